"""torch-facing wrappers of the C ABI: tensors in, tensors out.

PyTorch supplies device memory and the current stream; the three entry points
below only check shapes, allocate outputs and hand raw pointers to
libo1d.so.  theta is a float32 tensor of per-channel angles in degrees.
"""
from __future__ import annotations

import ctypes
import functools
import operator

import torch
from torch.autograd.function import once_differentiable

from . import _lib

_DT = {torch.float32: _lib.O1D_F32, torch.bfloat16: _lib.O1D_BF16}


# The current stream's handle without a Stream object around it (2 us less per call), where this torch has that.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor) -> int:
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _dt(t: torch.Tensor) -> int:
    if t.dtype not in _DT:
        raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")
    return _DT[t.dtype]


def _check_common(x: torch.Tensor, w: torch.Tensor, theta: torch.Tensor):
    if x.dim() != 4 or w.dim() != 2:
        raise ValueError("expected x as (N, C, H, W) and w as (C, K)")
    N, C, H, W = x.shape
    if w.shape[0] != C or theta.shape != (C,):
        raise ValueError(f"w {tuple(w.shape)} / theta {tuple(theta.shape)} do not match C={C}")
    if w.dtype != x.dtype:
        raise TypeError("x and w must share a dtype")
    if theta.dtype != torch.float32:
        raise TypeError("theta must be float32 degrees")
    for t in (x, w, theta):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous and on the GPU")
    return N, C, H, W, int(w.shape[1])


def _out(out: torch.Tensor | None, like: torch.Tensor, shape=None) -> torch.Tensor:
    """A caller-given output must match what the kernels write (they take no strides or sizes of it)."""
    shape = tuple(like.shape) if shape is None else tuple(shape)
    if out is None:
        return torch.empty(shape, dtype=like.dtype, device=like.device)
    if tuple(out.shape) != shape or out.dtype != like.dtype or out.device != like.device or not out.is_contiguous():
        raise ValueError(f"output {tuple(out.shape)} {out.dtype} {out.device} must be a contiguous {shape} "
                         f"{like.dtype} tensor on {like.device}")
    return out


def fwd(x: torch.Tensor, w: torch.Tensor, theta: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """y = oriented depthwise 1D convolution of x (Definition 1, Eq. 1-2)."""
    N, C, H, W, K = _check_common(x, w, theta)
    y = _out(out, x)
    _lib.check("o1d_fwd", _lib.call("o1d_fwd", x.data_ptr(), w.data_ptr(), theta.data_ptr(), y.data_ptr(),
                                    N, C, H, W, K, _dt(x), _stream(x)))
    return y


def bwd_input(dy: torch.Tensor, w: torch.Tensor, theta: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """dx given dy (adjoint of Eq. 1 in x)."""
    N, C, H, W, K = _check_common(dy, w, theta)
    dx = _out(out, dy)
    _lib.check("o1d_bwd_input", _lib.call("o1d_bwd_input", dy.data_ptr(), w.data_ptr(), theta.data_ptr(),
                                          dx.data_ptr(), N, C, H, W, K, _dt(dy), _stream(dy)))
    return dx


def workspace_bytes(N: int, C: int, H: int, W: int, K: int, dtype: torch.dtype) -> int:
    return int(_lib.lib().o1d_bwd_weight_workspace_bytes(N, C, H, W, K, _DT[dtype]))


def _workspace(workspace: torch.Tensor | None, like: torch.Tensor, need: int) -> tuple[torch.Tensor, int]:
    """A caller-given workspace must be device memory the kernels may write: a contiguous tensor on like's GPU
    holding at least `need` bytes."""
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=like.device)
    if not workspace.is_cuda or workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on {like.device}, got {workspace.device} "
                         f"(contiguous={workspace.is_contiguous()})")
    nbytes = workspace.numel() * workspace.element_size()
    if nbytes < need:
        raise ValueError(f"workspace holds {nbytes} bytes, {need} needed")
    return workspace, nbytes


def bwd_weight(x: torch.Tensor, dy: torch.Tensor, theta: torch.Tensor, K: int, out: torch.Tensor | None = None,
               workspace: torch.Tensor | None = None) -> torch.Tensor:
    """dw (C, K) given x and dy (adjoint of Eq. 1 in w)."""
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("x and dy must have the same shape and dtype")
    N, C, H, W = x.shape
    dw = _out(out, x, (C, K))
    _check_common(x, dw, theta)
    if not dy.is_cuda or not dy.is_contiguous():
        raise ValueError("tensors must be contiguous and on the GPU")
    workspace, nbytes = _workspace(workspace, x, workspace_bytes(N, C, H, W, K, x.dtype))
    _lib.check("o1d_bwd_weight", _lib.call("o1d_bwd_weight", x.data_ptr(), dy.data_ptr(), theta.data_ptr(),
                                           dw.data_ptr(), N, C, H, W, K, _dt(x), workspace.data_ptr(), nbytes,
                                           _stream(x)))
    return dw


def bwd(x: torch.Tensor, dy: torch.Tensor, w: torch.Tensor, theta: torch.Tensor,
        out: tuple[torch.Tensor, torch.Tensor] | None = None,
        workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """(dx, dw) given x and dy: both adjoints of Eq. 1 in one call."""
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("x and dy must have the same shape and dtype")
    N, C, H, W, K = _check_common(x, w, theta)
    if not dy.is_cuda or not dy.is_contiguous():
        raise ValueError("tensors must be contiguous and on the GPU")
    dx, dw = (_out(None, x), _out(None, w)) if out is None else (_out(out[0], x), _out(out[1], w))
    workspace, nbytes = _workspace(workspace, x, workspace_bytes(N, C, H, W, K, x.dtype))
    _lib.check("o1d_bwd", _lib.call("o1d_bwd", x.data_ptr(), dy.data_ptr(), w.data_ptr(), theta.data_ptr(),
                                    dx.data_ptr(), dw.data_ptr(), N, C, H, W, K, _dt(x), workspace.data_ptr(),
                                    nbytes, _stream(x)))
    return dx, dw


# ---------------------------------------------------------------- stride, layout, sampling

_LAYOUT = {"nchw": _lib.O1D_NCHW, "nhwc": _lib.O1D_NHWC}
_SAMPLING = {"floor": _lib.O1D_FLOOR, "bilinear": _lib.O1D_BILINEAR}


def out_size(n: int, stride: int) -> int:
    """Output length along one axis: floor((n - 1) / stride) + 1."""
    return (n - 1) // stride + 1


def _ex_args(x: torch.Tensor, w: torch.Tensor, theta: torch.Tensor, layout: str, sampling: str):
    if layout not in _LAYOUT or sampling not in _SAMPLING:
        raise ValueError(f"layout must be one of {list(_LAYOUT)}, sampling one of {list(_SAMPLING)}")
    if x.dim() != 4 or w.dim() != 2:
        raise ValueError("expected a 4-d x and w as (C, K)")
    if layout == "nchw":
        N, C, H, W = x.shape
    else:
        N, H, W, C = x.shape
    if w.shape[0] != C or theta.shape != (C,):
        raise ValueError(f"w {tuple(w.shape)} / theta {tuple(theta.shape)} do not match C={C}")
    if w.dtype != x.dtype:
        raise TypeError("x and w must share a dtype")
    if theta.dtype != torch.float32:
        raise TypeError("theta must be float32 degrees")
    for t in (x, w, theta):
        if not t.is_cuda or not t.is_contiguous() or t.device != x.device:
            raise ValueError("tensors must be contiguous and on one GPU")
    return N, C, H, W, int(w.shape[1])


def _shape(layout: str, N: int, C: int, H: int, W: int) -> tuple:
    return (N, C, H, W) if layout == "nchw" else (N, H, W, C)


def fwd_ex(x: torch.Tensor, w: torch.Tensor, theta: torch.Tensor, stride: int = 1, layout: str = "nchw",
           sampling: str = "floor", out: torch.Tensor | None = None) -> torch.Tensor:
    """Forward pass with stride, NCHW / NHWC layout and rounded-down or bilinear sampling."""
    N, C, H, W, K = _ex_args(x, w, theta, layout, sampling)
    y = _out(out, x, _shape(layout, N, C, out_size(H, stride), out_size(W, stride)))
    _lib.check("o1d_fwd_ex", _lib.call("o1d_fwd_ex", x.data_ptr(), w.data_ptr(), theta.data_ptr(), y.data_ptr(),
                                       N, C, H, W, K, stride, _LAYOUT[layout], _SAMPLING[sampling], _dt(x),
                                       _stream(x)))
    return y


def bwd_input_ex(dy: torch.Tensor, w: torch.Tensor, theta: torch.Tensor, in_hw: tuple[int, int], stride: int = 1,
                 layout: str = "nchw", sampling: str = "floor", out: torch.Tensor | None = None) -> torch.Tensor:
    """dx (input plane in_hw = (H, W)) given dy of the stride-`stride` output plane."""
    N, C, P, Q, K = _ex_args(dy, w, theta, layout, sampling)
    H, W = in_hw
    if (out_size(H, stride), out_size(W, stride)) != (P, Q):
        raise ValueError(f"dy plane {P}x{Q} is not the stride-{stride} output of {H}x{W}")
    dx = _out(out, dy, _shape(layout, N, C, H, W))
    _lib.check("o1d_bwd_input_ex", _lib.call("o1d_bwd_input_ex", dy.data_ptr(), w.data_ptr(), theta.data_ptr(),
                                             dx.data_ptr(), N, C, H, W, K, stride, _LAYOUT[layout],
                                             _SAMPLING[sampling], _dt(dy), _stream(dy)))
    return dx


def workspace_bytes_ex(N: int, C: int, H: int, W: int, K: int, dtype: torch.dtype, stride: int = 1,
                       layout: str = "nchw", sampling: str = "floor") -> int:
    return int(_lib.lib().o1d_bwd_weight_ex_workspace_bytes(N, C, H, W, K, stride, _LAYOUT[layout],
                                                            _SAMPLING[sampling], _DT[dtype]))


def bwd_weight_ex(x: torch.Tensor, dy: torch.Tensor, theta: torch.Tensor, K: int, stride: int = 1,
                  layout: str = "nchw", sampling: str = "floor", out: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None) -> torch.Tensor:
    """dw (C, K) given x and dy of the stride-`stride` output plane."""
    if layout not in _LAYOUT or sampling not in _SAMPLING:
        raise ValueError(f"layout must be one of {list(_LAYOUT)}, sampling one of {list(_SAMPLING)}")
    N, H, W, C = (x.shape[0], x.shape[1], x.shape[2], x.shape[3]) if layout == "nhwc" else \
        (x.shape[0], x.shape[2], x.shape[3], x.shape[1])
    if tuple(dy.shape) != _shape(layout, N, C, out_size(H, stride), out_size(W, stride)) or dy.dtype != x.dtype:
        raise ValueError(f"dy {tuple(dy.shape)} does not match x {tuple(x.shape)} at stride {stride}")
    dw = _out(out, x, (C, K))
    _ex_args(x, dw, theta, layout, sampling)
    if not dy.is_cuda or not dy.is_contiguous() or dy.device != x.device:
        raise ValueError("tensors must be contiguous and on one GPU")
    workspace, nbytes = _workspace(workspace, x, workspace_bytes_ex(N, C, H, W, K, x.dtype, stride, layout, sampling))
    _lib.check("o1d_bwd_weight_ex", _lib.call("o1d_bwd_weight_ex", x.data_ptr(), dy.data_ptr(), theta.data_ptr(),
                                              dw.data_ptr(), N, C, H, W, K, stride, _LAYOUT[layout],
                                              _SAMPLING[sampling], _dt(x), workspace.data_ptr(), nbytes,
                                              _stream(x)))
    return dw


class OrientedConv1dFunction(torch.autograd.Function):
    """Autograd glue: forward -> o1d_fwd, backward -> o1d_bwd (or one of its halves); theta gets no gradient."""

    @staticmethod
    def forward(ctx, x, w, theta):
        # the kernels take dense tensors: save the dense copies that the forward used
        x, w, theta = x.contiguous(), w.contiguous(), theta.contiguous()
        ctx.save_for_backward(x, w, theta)
        return fwd(x, w, theta)

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, w, theta = ctx.saved_tensors
        gy = gy.contiguous()
        if ctx.needs_input_grad[0] and ctx.needs_input_grad[1]:
            gx, gw = bwd(x, gy, w, theta)
            return gx, gw, None
        gx = bwd_input(gy, w, theta) if ctx.needs_input_grad[0] else None
        gw = bwd_weight(x, gy, theta, w.shape[1]) if ctx.needs_input_grad[1] else None
        return gx, gw, None


# ---------------------------------------------------------------- depthwise separable block

def _check_pw(w_pw: torch.Tensor, like: torch.Tensor, C: int) -> int:
    if w_pw.dim() != 2 or w_pw.shape[1] != C or w_pw.dtype != like.dtype:
        raise ValueError(f"w_pw must be (C', {C}) of dtype {like.dtype}, got {tuple(w_pw.shape)} {w_pw.dtype}")
    if not w_pw.is_cuda or not w_pw.is_contiguous():
        raise ValueError("tensors must be contiguous and on the GPU")
    return int(w_pw.shape[0])


def dsc_fwd(x: torch.Tensor, w_dw: torch.Tensor, theta: torch.Tensor, w_pw: torch.Tensor,
            out: tuple[torch.Tensor, torch.Tensor] | None = None) -> tuple[torch.Tensor, torch.Tensor]:
    """(z, y): z the oriented depthwise convolution of x, y = w_pw mixing z's channels (Sec. 3.2, Table 1)."""
    N, C, H, W, K = _check_common(x, w_dw, theta)
    Co = _check_pw(w_pw, x, C)
    z, y = (_out(None, x), _out(None, x, (N, Co, H, W))) if out is None else \
        (_out(out[0], x), _out(out[1], x, (N, Co, H, W)))
    _lib.check("o1d_dsc_fwd", _lib.call("o1d_dsc_fwd", x.data_ptr(), w_dw.data_ptr(), theta.data_ptr(),
                                        w_pw.data_ptr(), z.data_ptr(), y.data_ptr(), N, C, Co, H, W, K, _dt(x),
                                        _stream(x)))
    return z, y


def dsc_workspace_bytes(N: int, C: int, Co: int, H: int, W: int, K: int, dtype: torch.dtype) -> int:
    return int(_lib.lib().o1d_dsc_bwd_workspace_bytes(N, C, Co, H, W, K, _DT[dtype]))


def dsc_bwd(x: torch.Tensor, z: torch.Tensor, dy: torch.Tensor, w_dw: torch.Tensor, theta: torch.Tensor,
            w_pw: torch.Tensor, out: tuple[torch.Tensor, torch.Tensor, torch.Tensor] | None = None,
            workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dw_dw, dw_pw) of the block given x, the forward's z and dy."""
    N, C, H, W, K = _check_common(x, w_dw, theta)
    Co = _check_pw(w_pw, x, C)
    if z.shape != x.shape or z.dtype != x.dtype or dy.shape != (N, Co, H, W) or dy.dtype != x.dtype:
        raise ValueError("z must match x, dy must be (N, C', H, W) of x's dtype")
    for t in (z, dy):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("tensors must be contiguous and on the GPU")
    if out is None:
        dx, dwd, dwp = _out(None, x), _out(None, w_dw), _out(None, w_pw)
    else:
        dx, dwd, dwp = _out(out[0], x), _out(out[1], w_dw), _out(out[2], w_pw)
    workspace, nbytes = _workspace(workspace, x, dsc_workspace_bytes(N, C, Co, H, W, K, x.dtype))
    _lib.check("o1d_dsc_bwd", _lib.call("o1d_dsc_bwd", x.data_ptr(), z.data_ptr(), dy.data_ptr(), w_dw.data_ptr(),
                                        theta.data_ptr(), w_pw.data_ptr(), dx.data_ptr(), dwd.data_ptr(),
                                        dwp.data_ptr(), N, C, Co, H, W, K, _dt(x), workspace.data_ptr(), nbytes,
                                        _stream(x)))
    return dx, dwd, dwp


# ---------------------------------------------------------------- row operators (channels last)
#
# An activation is any tensor whose last axis holds the features and whose other axes collapse to rows a fixed stride
# apart: a dense (N, H, W, C) tensor, an (M, C) matrix, or a slice of a wider one.

_bound = None
_BOUND = ("o1d_ln_fwd", "o1d_ln_bwd", "o1d_ln_bwd_workspace_bytes", "o1d_linear_fwd", "o1d_linear_bwd_input",
          "o1d_linear_bwd_weight", "o1d_linear_bwd_weight_workspace_bytes", "o1d_pack", "o1d_unpack")


def _direct():
    """The native calls of the common case (contiguous tensors that match, outputs made by the call); each returns None
    where it is another, which the checked code below takes."""
    global _bound
    if _bound is None:
        try:
            from . import _rows as native
        except ImportError as e:
            raise ImportError(f"{e}; build it with `python -m paper_2309_15812_amd.build`") from None
        lib = _lib.lib()
        native.bind(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _BOUND))
        _bound = native
    return _bound


def _rows(t: torch.Tensor, what: str) -> tuple[torch.Tensor, int, int, int]:
    """(t or a view of it that starts where it does, rows, features, row stride); refuses what the kernels cannot
    address."""
    C = t.shape[-1] if t.dim() else 0
    if C < 1:
        raise ValueError(f"{what} must have at least one feature on its last axis, got {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{what} must be on the GPU")
    if t.is_contiguous():
        return t, t.numel() // C, C, C
    try:
        v = t.view(-1, C) if t.numel() else t.reshape(0, C)
    except RuntimeError:
        raise ValueError(f"{what} {tuple(t.shape)} with strides {t.stride()} is no matrix of rows") from None
    M = v.shape[0]
    ld = v.stride(0) if M > 1 else C
    if (C > 1 and v.stride(1) != 1) or ld < C:
        raise ValueError(f"{what} {tuple(t.shape)} with strides {t.stride()} needs contiguous features and rows that do "
                         f"not overlap")
    return v, M, C, ld


def _run(fn: str, like: torch.Tensor, *args) -> None:
    """The C entry point on the current stream of like's device."""
    f, device = getattr(_lib.lib(), fn), like.get_device()
    if device == torch.cuda.current_device():
        status = f(*args, _stream(like))
    else:  # (the default stream's handle means the current device's)
        with torch.cuda.device(device):
            status = f(*args, _stream(like))
    if status:
        _lib.check(fn, status)


def _vector(t: torch.Tensor, what: str, C: int, like: torch.Tensor) -> torch.Tensor:
    if t.dim() != 1 or t.numel() != C or t.dtype is not like.dtype or t.get_device() != like.get_device() \
            or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous ({C},) tensor of {like.dtype} on {like.device}, got "
                         f"{tuple(t.shape)} {t.dtype} {t.device}")
    return t


def _weight(w: torch.Tensor, like: torch.Tensor) -> tuple[int, int]:
    if w.dim() != 2 or w.dtype is not like.dtype or w.get_device() != like.get_device() or not w.is_contiguous():
        raise ValueError(f"w must be a contiguous (O, I) tensor of {like.dtype} on {like.device}, got {tuple(w.shape)} "
                         f"{w.dtype} {w.device}")
    return int(w.shape[0]), int(w.shape[1])


def _act(act: str) -> int:
    if act not in _lib.ACT:
        raise ValueError(f"act must be one of {list(_lib.ACT)}, got {act!r}")
    return _lib.ACT[act]


def _same(t: torch.Tensor, what: str, M: int, C: int, like: torch.Tensor) -> tuple[torch.Tensor, int]:
    """t as rows, checked to be M x C like `like`; (t, row stride)."""
    if t.dtype is not like.dtype or t.get_device() != like.get_device():
        raise ValueError(f"{what} must be {like.dtype} on {like.device}, got {t.dtype} on {t.device}")
    v, m, c, ld = _rows(t, what)
    if (m, c) != (M, C):
        raise ValueError(f"{what} has {m} rows of {c} features, expected {M} of {C}")
    return v, ld


class Packed8:
    """An 8-bit checkpoint of rows of `cols` features: int8 `q` (M, cols rounded up to 16) and float32 `scale`
    (M, ceil(cols / 64)); group g of a row stands for q[64 g : 64 g + 64] * scale[g]."""

    __slots__ = ("q", "scale", "cols")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, cols: int):
        ldq, groups = -(-cols // 16) * 16, -(-cols // _lib.GROUP)
        if cols < 1 or q.dim() != 2 or q.dtype != torch.int8 or q.shape[1] != ldq or not q.is_contiguous():
            raise ValueError(f"q must be a contiguous int8 (M, {ldq}) tensor, got {tuple(q.shape)} {q.dtype}")
        if scale.shape != (q.shape[0], groups) or scale.dtype != torch.float32 or not scale.is_contiguous():
            raise ValueError(f"scale must be a contiguous float32 ({q.shape[0]}, {groups}) tensor, got "
                             f"{tuple(scale.shape)} {scale.dtype}")
        if not q.is_cuda or q.device != scale.device:
            raise ValueError("a checkpoint's tensors must be on one GPU")
        self.q, self.scale, self.cols = q, scale, cols

    @staticmethod
    def of(q: torch.Tensor, scale: torch.Tensor, cols: int) -> "Packed8":  # (tensors made for it)
        held = object.__new__(Packed8)
        held.q, held.scale, held.cols = q, scale, cols
        return held

    @staticmethod
    def empty(M: int, cols: int, device) -> "Packed8":
        return Packed8.of(torch.empty((M, -(-cols // 16) * 16), dtype=torch.int8, device=device),
                          torch.empty((M, -(-cols // _lib.GROUP)), dtype=torch.float32, device=device), cols)

    @property
    def rows(self) -> int:
        return int(self.q.shape[0])

    @property
    def nbytes(self) -> int:
        return self.q.numel() + 4 * self.scale.numel()


def _either(t, what: str, M: int, C: int, like: torch.Tensor) -> tuple:
    """(pointer, row stride, q, scale) of a tensor or a checkpoint of M rows of C features."""
    if isinstance(t, Packed8):
        if t.cols != C or t.q.shape[0] != M or t.q.get_device() != like.get_device():
            raise ValueError(f"{what} is a checkpoint of {t.rows} rows of {t.cols} features on {t.q.device}, expected "
                             f"{M} of {C} on {like.device}")
        return None, C, t.q.data_ptr(), t.scale.data_ptr()
    v, ld = _same(t, what, M, C, like)
    return v.data_ptr(), ld, None, None


def _into(out: torch.Tensor | None, like: torch.Tensor, C: int) -> torch.Tensor:
    """Output with like's leading axes and C features."""
    shape = like.shape
    if out is not None:
        return _out(out, like, (*shape[:-1], C))
    return torch.empty_like(like) if shape[-1] == C and like.is_contiguous() else like.new_empty((*shape[:-1], C))


# What a call that uses no workspace asks for: it writes nothing there, so one tensor serves all such calls on all streams.
# Calls that write to theirs ask for 512 bytes at least.
_NO_SPACE = 256
_no_space: dict[int, torch.Tensor] = {}


def _scratch(workspace: torch.Tensor | None, like: torch.Tensor, need: int) -> tuple[torch.Tensor, int]:
    if workspace is not None:
        return _workspace(workspace, like, need)
    if need > _NO_SPACE:
        return like.new_empty((need,), dtype=torch.uint8), need
    held = _no_space.get(like.get_device())
    if held is None:
        held = _no_space[like.get_device()] = torch.empty((_NO_SPACE,), dtype=torch.uint8, device=like.device)
    return held, _NO_SPACE


def pack8(x: torch.Tensor) -> Packed8:
    """The 8-bit checkpoint of x's rows."""
    made = _direct().pack8(x)
    if made is not None:
        return Packed8.of(*made, x.shape[-1])
    dt = _dt(x)
    v, M, C, ld = _rows(x, "x")
    held = Packed8.empty(M, C, x.device)
    _run("o1d_pack", x, v.data_ptr(), ld, held.q.data_ptr(), held.scale.data_ptr(), M, C, dt)
    return held


def unpack8(held: Packed8, dtype: torch.dtype, act: str = "none", out: torch.Tensor | None = None) -> torch.Tensor:
    """act(what a checkpoint stands for), as (M, cols) of dtype."""
    if dtype not in _DT:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    if out is None:
        y = _direct().unpack8(held.q, held.scale, held.cols, _DT[dtype], _act(act))
        if y is not None:
            return y
    if out is None:
        y = v = torch.empty((held.rows, held.cols), dtype=dtype, device=held.q.device)
        ld = held.cols
    else:
        if out.dtype != dtype or out.device != held.q.device:
            raise ValueError(f"out must be {dtype} on {held.q.device}")
        y = out
        v, ld = _same(out, "out", held.rows, held.cols, out)
    _run("o1d_unpack", held.q, held.q.data_ptr(), held.scale.data_ptr(), _act(act), v.data_ptr(), ld, held.rows, held.cols,
         _DT[dtype])
    return y


def ln_fwd(x: torch.Tensor, w: torch.Tensor, b: torch.Tensor, eps: float = 1e-6, out: torch.Tensor | None = None
           ) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(y, mean, rstd): layer norm over the last axis; mean and rstd (M,) float32 are for ln_bwd."""
    if out is None:
        made = _direct().ln_fwd(x, w, b, eps)
        if made is not None:
            return made
    dt = _dt(x)
    v, M, C, ld = _rows(x, "x")
    _vector(w, "w", C, x)
    _vector(b, "b", C, x)
    y = _into(out, x, C)
    mean, rstd = x.new_empty((M,), dtype=torch.float32), x.new_empty((M,), dtype=torch.float32)
    _run("o1d_ln_fwd", x, v.data_ptr(), ld, w.data_ptr(), b.data_ptr(), y.data_ptr(), C, mean.data_ptr(), rstd.data_ptr(),
         M, C, eps, dt)
    return y, mean, rstd


@functools.lru_cache(maxsize=4096)
def ln_workspace_bytes(M: int, C: int, dtype: torch.dtype) -> int:
    return int(_lib.lib().o1d_ln_bwd_workspace_bytes(M, C, _DT[dtype]))


def ln_bwd(x: torch.Tensor | Packed8, dy: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, w: torch.Tensor,
           out: tuple[torch.Tensor, torch.Tensor, torch.Tensor] | None = None,
           workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dw, db) of ln_fwd given its input (or the input's checkpoint), dy and its mean and rstd."""
    if out is None and workspace is None:
        held = isinstance(x, Packed8)
        made = _direct().ln_bwd(x.q if held else x, x.scale if held else None, x.cols if held else 0, dy, mean, rstd, w)
        if made is not None:
            return made
    dt = _dt(dy)
    g, M, C, lddy = _rows(dy, "dy")
    px, ldx, q, scale = _either(x, "x", M, C, dy)
    _vector(w, "w", C, dy)
    for t, n in ((mean, "mean"), (rstd, "rstd")):
        if t.dim() != 1 or t.numel() != M or t.dtype is not torch.float32 or t.get_device() != dy.get_device() \
                or not t.is_contiguous():
            raise ValueError(f"{n} must be a contiguous float32 ({M},) tensor on {dy.device}")
    dx, dw, db = (None, None, None) if out is None else out
    dx = _into(dx, dy, C)
    dw, db = (torch.empty_like(w) if t is None else _out(t, w) for t in (dw, db))
    workspace, nbytes = _scratch(workspace, dy, ln_workspace_bytes(M, C, dy.dtype))
    _run("o1d_ln_bwd", dy, px, ldx, q, scale, g.data_ptr(), lddy, mean.data_ptr(), rstd.data_ptr(), w.data_ptr(),
         dx.data_ptr(), C, dw.data_ptr(), db.data_ptr(), M, C, dt, workspace.data_ptr(), nbytes)
    return dx, dw, db


def linear_fwd(x: torch.Tensor, w: torch.Tensor, b: torch.Tensor | None = None, act: str = "none",
               residual: torch.Tensor | None = None, save: str | None = None, out: torch.Tensor | None = None):
    """y = act(x w^T + b) + residual for w (O, I).  save="pre" returns (y, pre) with the pre-activation x w^T + b as a
    tensor, save="pack8" returns (y, its checkpoint)."""
    if save not in (None, "pre", "pack8"):
        raise ValueError(f"save must be None, 'pre' or 'pack8', got {save!r}")
    a = _act(act)
    if out is None:
        made = _direct().linear_fwd(x, w, b, a, residual, 0 if save is None else 1 if save == "pre" else 2)
        if made is not None:
            return made if save != "pack8" else (made[0], Packed8.of(made[1], made[2], w.shape[0]))
    dt = _dt(x)
    v, M, I, ldx = _rows(x, "x")
    O, wi = _weight(w, x)
    if wi != I:
        raise ValueError(f"w {tuple(w.shape)} does not take {I} features")
    if b is not None:
        _vector(b, "b", O, x)
    res, ldres = (None, O) if residual is None else _same(residual, "residual", M, O, x)
    y = _into(out, x, O)
    pre = _into(None, x, O) if save == "pre" else None
    held = Packed8.empty(M, O, x.device) if save == "pack8" else None
    _run("o1d_linear_fwd", x, v.data_ptr(), ldx, w.data_ptr(), None if b is None else b.data_ptr(), a,
         None if res is None else res.data_ptr(), ldres, y.data_ptr(), O, None if pre is None else pre.data_ptr(), O,
         None if held is None else held.q.data_ptr(), None if held is None else held.scale.data_ptr(), M, I, O, dt)
    return y if save is None else (y, pre if held is None else held)


def linear_bwd_input(dy: torch.Tensor, w: torch.Tensor, pre: torch.Tensor | Packed8 | None = None, act: str = "none",
                     out: torch.Tensor | None = None) -> torch.Tensor:
    """dx = (dy w) act'(pre): the gradient in a product's input, carried through the activation that made it
    (pre: that activation's argument, a tensor or a checkpoint)."""
    a = _act(act)
    if out is None:
        held = isinstance(pre, Packed8)
        made = _direct().linear_bwd_input(dy, w, pre.q if held else pre, pre.scale if held else None,
                                          pre.cols if held else 0, a)
        if made is not None:
            return made
    dt = _dt(dy)
    g, M, O, lddy = _rows(dy, "dy")
    wo, I = _weight(w, dy)
    if wo != O:
        raise ValueError(f"w {tuple(w.shape)} does not give {O} features")
    if (pre is None) != (act == "none"):
        raise ValueError("pre and act are given together")
    p, ldp, q, scale = (None, I, None, None) if pre is None else _either(pre, "pre", M, I, dy)
    dx = _into(out, dy, I)
    _run("o1d_linear_bwd_input", dy, g.data_ptr(), lddy, w.data_ptr(), a, p, ldp, q, scale, dx.data_ptr(), I, M, I, O, dt)
    return dx


@functools.lru_cache(maxsize=4096)
def linear_workspace_bytes(M: int, I: int, O: int, dtype: torch.dtype, act: str = "none", packed: bool = False) -> int:
    return int(_lib.lib().o1d_linear_bwd_weight_workspace_bytes(M, I, O, _act(act), int(packed), _DT[dtype]))


def linear_bwd_weight(x: torch.Tensor | Packed8, dy: torch.Tensor, act: str = "none", bias: bool = True,
                      out: tuple[torch.Tensor, torch.Tensor | None] | None = None,
                      workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor | None]:
    """(dw, db): dw (O, I) = dy^T act(x), db = dy's sum over rows (None with bias=False).  x is the product's input, or
    (with act) the pre-activation that it was made from, as a tensor or a checkpoint."""
    a, held = _act(act), isinstance(x, Packed8)
    I = x.cols if held else int(x.shape[-1]) if x.dim() else 0
    if out is None and workspace is None:
        made = _direct().linear_bwd_weight(x.q if held else x, x.scale if held else None, I, dy, a, bias)
        if made is not None:
            return made
    dt = _dt(dy)
    g, M, O, lddy = _rows(dy, "dy")
    p, ldx, q, scale = _either(x, "x", M, I, dy)
    dw, db = (None, None) if out is None else out
    dw = dy.new_empty((O, I)) if dw is None else _out(dw, dy, (O, I))
    db = None if not bias else dy.new_empty((O,)) if db is None else _out(db, dy, (O,))
    workspace, nbytes = _scratch(workspace, dy, linear_workspace_bytes(M, I, O, dy.dtype, act, q is not None))
    _run("o1d_linear_bwd_weight", dy, p, ldx, q, scale, a, g.data_ptr(), lddy, dw.data_ptr(),
         None if db is None else db.data_ptr(), M, I, O, dt, workspace.data_ptr(), nbytes)
    return dw, db


def act_bwd(pre: torch.Tensor | Packed8, dy: torch.Tensor, act: str, out: torch.Tensor | None = None) -> torch.Tensor:
    """dh = dy act'(pre), pre a tensor or a checkpoint."""
    dt, a = _dt(dy), _act(act)
    g, M, C, lddy = _rows(dy, "dy")
    p, ldp, q, scale = _either(pre, "pre", M, C, dy)
    dh = _into(out, dy, C)
    _run("o1d_act_bwd", dy, p, ldp, q, scale, a, g.data_ptr(), lddy, dh.data_ptr(), C, M, C, dt)
    return dh


class LayerNormFunction(torch.autograd.Function):
    """Autograd glue: ln_fwd, ln_bwd.  checkpoint=True keeps x in 8 bits for the backward."""

    @staticmethod
    def forward(ctx, x, w, b, eps=1e-6, checkpoint=False):
        x, w, b = x.contiguous(), w.contiguous(), b.contiguous()
        y, mean, rstd = ln_fwd(x, w, b, eps)
        held = pack8(x) if checkpoint else None
        ctx.cols = x.shape[-1]
        ctx.save_for_backward(*((held.q, held.scale) if checkpoint else (x, None)), mean, rstd, w)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, scale, mean, rstd, w = ctx.saved_tensors
        gx, gw, gb = ln_bwd(x if scale is None else Packed8(x, scale, ctx.cols), gy.contiguous(), mean, rstd, w)
        return gx, gw, gb, None, None


class LinearFunction(torch.autograd.Function):
    """Autograd glue: y = act(x w^T + b) + residual.  checkpoint=True keeps x and the pre-activation in 8 bits for the
    backward."""

    @staticmethod
    def forward(ctx, x, w, b=None, act="none", residual=None, checkpoint=False):
        x, w = x.contiguous(), w.contiguous()
        save = None if act == "none" else "pack8" if checkpoint else "pre"
        out = linear_fwd(x, w, None if b is None else b.contiguous(), act,
                         None if residual is None else residual.contiguous(), save)
        y, pre = (out, None) if save is None else out
        ctx.act, ctx.bias = act, b is not None
        ctx.residual = None if residual is None else residual.shape  # (its leading axes may be others)
        ctx.save_for_backward(w, *_parts(pack8(x) if checkpoint else x), *_parts(pre))
        ctx.cols = (w.shape[1], w.shape[0])
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        w, x, xs, pre, ps = ctx.saved_tensors
        dy = gy.contiguous()
        dh = dy if ctx.act == "none" else act_bwd(_whole(pre, ps, ctx.cols[1]), dy, ctx.act)
        wants = (*ctx.needs_input_grad, False, False, False)  # (arguments left out have no entry)
        gx = linear_bwd_input(dh, w) if wants[0] else None
        gw = gb = None
        if wants[1] or (ctx.bias and wants[2]):
            gw, gb = linear_bwd_weight(_whole(x, xs, ctx.cols[0]), dh, bias=ctx.bias)
        return gx, gw, gb, None, (gy.reshape(ctx.residual) if wants[4] else None), None


def _parts(t) -> tuple:
    """A tensor, a checkpoint or None as two tensors (or None) that autograd can save."""
    return (t.q, t.scale) if isinstance(t, Packed8) else (t, None)


def _whole(t, scale, cols: int):
    return t if scale is None else Packed8(t, scale, cols)


# ---------------------------------------------------------------- group norm with an activation (channels last)

def _samples(t: torch.Tensor, what: str) -> tuple[torch.Tensor, int, int, int, int]:
    """(t or a view of it, samples, pixels of one, channels, row stride) of a tensor (N, ..., C)."""
    if t.dim() < 2:
        raise ValueError(f"{what} must be (N, ..., C), got {tuple(t.shape)}")
    v, M, C, ld = _rows(t, what)
    N = int(t.shape[0])
    if N and not M:
        raise ValueError(f"{what} {tuple(t.shape)} has samples without pixels")
    return v, N, M // N if N else 0, C, ld


def _stats(t: torch.Tensor, what: str, shape: tuple[int, int] | None, like: torch.Tensor) -> torch.Tensor:
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != shape) or t.dtype is not torch.float32 \
            or t.get_device() != like.get_device() or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous float32 (N, groups) tensor on {like.device}, got {tuple(t.shape)} "
                         f"{t.dtype} {t.device}")
    return t


@functools.lru_cache(maxsize=4096)
def gn_workspace_bytes(N: int, P: int, C: int, groups: int, dtype: torch.dtype, backward: bool) -> int:
    f = _lib.lib().o1d_gn_bwd_workspace_bytes if backward else _lib.lib().o1d_gn_fwd_workspace_bytes
    return int(f(N, P, C, groups, _DT[dtype]))


_bound_train = None
_BOUND_TRAIN = ("o1d_gn_fwd", "o1d_gn_fwd_workspace_bytes", "o1d_gn_bwd", "o1d_gn_bwd_workspace_bytes", "o1d_pack_scaled",
                "o1d_pack_scaled_workspace_bytes", "o1d_scaled_linear_fwd", "o1d_scaled_linear_bwd_input",
                "o1d_scaled_linear_bwd_weight", "o1d_scaled_linear_bwd_weight_workspace_bytes", "o1d_adamw",
                "o1d_adamw_workspace_bytes")


def _train():
    """The native calls of the common case of what follows; each returns None where it is another."""
    global _bound_train
    if _bound_train is None:
        try:
            from . import _train as native
        except ImportError as e:
            raise ImportError(f"{e}; build it with `python -m paper_2309_15812_amd.build`") from None
        lib = _lib.lib()
        native.bind(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _BOUND_TRAIN))
        _bound_train = native
    return _bound_train


def gn_fwd(x: torch.Tensor, w: torch.Tensor, b: torch.Tensor, groups: int, eps: float = 1e-5, act: str = "none",
           out: torch.Tensor | None = None, workspace: torch.Tensor | None = None
           ) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(y, mean, rstd): act of the group norm of x (N, ..., C) over a sample's pixels and the C / groups channels of a group;
    mean and rstd (N, groups) float32 are for gn_bwd."""
    a, groups = _act(act), operator.index(groups)
    if out is None and workspace is None:
        made = _train().gn_fwd(x, w, b, groups, eps, a)
        if made is not None:
            return made
    dt = _dt(x)
    v, N, P, C, ld = _samples(x, "x")
    _vector(w, "w", C, x)
    _vector(b, "b", C, x)
    if groups < 1 or C % groups:
        raise ValueError(f"groups={groups} do not divide {C} channels")
    y = _into(out, x, C)
    mean, rstd = (x.new_empty((N, groups), dtype=torch.float32) for _ in range(2))
    workspace, nbytes = _scratch(workspace, x, gn_workspace_bytes(N, P, C, groups, x.dtype, False))
    _run("o1d_gn_fwd", x, v.data_ptr(), ld, w.data_ptr(), b.data_ptr(), a, y.data_ptr(), C, mean.data_ptr(),
         rstd.data_ptr(), N, P, C, groups, eps, dt, workspace.data_ptr(), nbytes)
    return y, mean, rstd


def gn_bwd(x: torch.Tensor, dy: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, w: torch.Tensor, b: torch.Tensor,
           act: str = "none", out: tuple[torch.Tensor, torch.Tensor, torch.Tensor] | None = None,
           workspace: torch.Tensor | None = None) -> tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dw, db) of gn_fwd given its input, dy and its mean and rstd."""
    a = _act(act)
    if out is None and workspace is None:
        made = _train().gn_bwd(x, dy, mean, rstd, w, b, a)
        if made is not None:
            return made
    dt = _dt(dy)
    g, N, P, C, lddy = _samples(dy, "dy")
    v, ldx = _same(x, "x", N * P, C, dy)
    _stats(mean, "mean", None, dy)
    groups = int(mean.shape[1])
    _stats(rstd, "rstd", (N, groups), dy)
    _stats(mean, "mean", (N, groups), dy)
    _vector(w, "w", C, dy)
    _vector(b, "b", C, dy)
    if groups < 1 or C % groups:
        raise ValueError(f"{groups} groups of the statistics do not divide {C} channels")
    dx, dw, db = (None, None, None) if out is None else out
    dx = _into(dx, dy, C)
    dw, db = (torch.empty_like(w) if t is None else _out(t, w) for t in (dw, db))
    workspace, nbytes = _scratch(workspace, dy, gn_workspace_bytes(N, P, C, groups, dy.dtype, True))
    _run("o1d_gn_bwd", dy, v.data_ptr(), ldx, g.data_ptr(), lddy, mean.data_ptr(), rstd.data_ptr(), w.data_ptr(),
         b.data_ptr(), a, dx.data_ptr(), C, dw.data_ptr(), db.data_ptr(), N, P, C, groups, dt, workspace.data_ptr(), nbytes)
    return dx, dw, db


class GroupNormFunction(torch.autograd.Function):
    """Autograd glue: gn_fwd, gn_bwd."""

    @staticmethod
    def forward(ctx, x, w, b, groups, eps=1e-5, act="none"):
        x, w, b = x.contiguous(), w.contiguous(), b.contiguous()
        y, mean, rstd = gn_fwd(x, w, b, groups, eps, act)
        ctx.act = act
        ctx.save_for_backward(x, mean, rstd, w, b)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, mean, rstd, w, b = ctx.saved_tensors
        gx, gw, gb = gn_bwd(x, gy.contiguous(), mean, rstd, w, b, ctx.act)
        return gx, gw, gb, None, None, None


# ---------------------------------------------------------------- products of 8-bit floating point operands

_F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_F8_OF = {t: _lib.SCALED[n] for n, t in _F8.items()}
_ALONG = {"features": 1, "rows": 2, "both": 3}


class F8:
    """A matrix of rows of `cols` values in 8-bit floating point with a power-of-two scale for each 128 values of a row: q
    (R, cols rounded up to 128) float8_e4m3fn or float8_e5m2, zeros behind a row's end, and exponents e (ceil(cols / 128), R
    rounded up to 16) uint8; q[r, k] 2^(e[k / 128, r] - 127) is the value."""

    __slots__ = ("q", "e", "cols")

    def __init__(self, q: torch.Tensor, e: torch.Tensor, cols: int):
        cols = operator.index(cols)
        groups = -(-cols // _lib.SCALED_GROUP)
        if cols < 1 or q.dim() != 2 or q.dtype not in _F8_OF or q.shape[1] != groups * _lib.SCALED_GROUP \
                or not q.is_contiguous():
            raise ValueError(f"q must be a contiguous (R, {groups * _lib.SCALED_GROUP}) tensor of float8_e4m3fn or "
                             f"float8_e5m2, got {tuple(q.shape)} {q.dtype}")
        if tuple(e.shape) != (groups, -(-q.shape[0] // 16) * 16) or e.dtype != torch.uint8 or not e.is_contiguous():
            raise ValueError(f"e must be a contiguous uint8 ({groups}, {-(-q.shape[0] // 16) * 16}) tensor, got "
                             f"{tuple(e.shape)} {e.dtype}")
        if not q.is_cuda or q.device != e.device:
            raise ValueError("an operand's tensors must be on one GPU")
        self.q, self.e, self.cols = q, e, cols

    @staticmethod
    def of(q: torch.Tensor, e: torch.Tensor, cols: int) -> "F8":  # (tensors made for it)
        held = object.__new__(F8)
        held.q, held.e, held.cols = q, e, cols
        return held

    @staticmethod
    def empty(R: int, cols: int, fmt: str, device) -> "F8":
        groups = -(-cols // _lib.SCALED_GROUP)
        return F8.of(torch.empty((R, groups * _lib.SCALED_GROUP), dtype=_F8[fmt], device=device),
                     torch.empty((groups, -(-R // 16) * 16), dtype=torch.uint8, device=device), cols)

    @property
    def rows(self) -> int:
        return int(self.q.shape[0])

    @property
    def nbytes(self) -> int:
        return self.q.numel() + self.e.numel()

    def float(self) -> torch.Tensor:
        """What it stands for, in float32 (by torch: for looking at, not for computing with)."""
        e = self.e[:, :self.rows].to(torch.int32)
        # (a float32's exponent field is the same number; 0 stands for 2^-127, which has a fraction's bit instead, 255 for NaN)
        bits = torch.where(e == 0, 1 << 22, torch.where(e == 255, 0x7fc00000, e << 23))
        scale = bits.to(torch.int32).view(torch.float32).t().repeat_interleave(_lib.SCALED_GROUP, 1)
        return (self.q.float() * scale)[:, :self.cols]


def _f8(t: F8, what: str, R: int | None, cols: int, like: torch.Tensor, second: bool = False) -> F8:
    if not isinstance(t, F8):
        raise TypeError(f"{what} must be packed (pack_f8), got {type(t).__name__}")
    if t.cols != cols or (R is not None and t.rows != R) or t.q.get_device() != like.get_device():
        raise ValueError(f"{what} has {t.rows} rows of {t.cols} values on {t.q.device}, expected "
                         f"{'' if R is None else R} rows of {cols} on {like.device}")
    if second and t.q.dtype is not torch.float8_e4m3fn:
        raise TypeError(f"{what} must be e4m3, got {t.q.dtype}")
    return t


def pack_f8(x: torch.Tensor, fmt: str = "e4m3", along: str = "features", sums: bool = False,
            workspace: torch.Tensor | None = None):
    """x's rows as 8-bit operands of products that sum along: "features" -> F8 of (M, C); "rows" -> F8 of x transposed
    (C, M), "both" -> the two.  sums=True (not with "features" alone) appends the columns' sums, a bias gradient, in
    x's type."""
    if fmt not in _F8 or along not in _ALONG:
        raise ValueError(f"fmt must be one of {list(_F8)}, along 'features', 'rows' or 'both'; got {fmt!r}, {along!r}")
    if sums and along == "features":
        raise ValueError("sums come with along='rows' or 'both'")
    if workspace is None:
        made = _train().pack(x, _lib.SCALED[fmt], _ALONG[along], bool(sums))
        if made is not None:
            C = x.shape[-1]
            if along == "features":
                return F8.of(*made, C)
            M = x.numel() // C
            if along == "rows":
                return (F8.of(made[0], made[1], M), made[2]) if sums else F8.of(*made, M)
            return (F8.of(made[0], made[1], C), F8.of(made[2], made[3], M), *made[4:])
    dt = _dt(x)
    v, M, C, ld = _rows(x, "x")
    r = F8.empty(M, C, fmt, x.device) if along != "rows" else None
    t = None
    if along != "features":
        if M < 1:
            raise ValueError("no rows to sum along")
        t = F8.empty(C, M, fmt, x.device)
    total = x.new_empty((C,)) if sums else None
    pw, nbytes = None, 0
    if sums:
        workspace, nbytes = _scratch(workspace, x, int(_lib.lib().o1d_pack_scaled_workspace_bytes(M, C, 1)))
        pw = workspace.data_ptr()
    _run("o1d_pack_scaled", x, v.data_ptr(), ld, _lib.SCALED[fmt], *((r.q.data_ptr(), r.e.data_ptr()) if r else (None, None)),
         *((t.q.data_ptr(), t.e.data_ptr()) if t else (None, None)), None if total is None else total.data_ptr(), M, C, dt,
         pw, nbytes)
    got = tuple(k for k in (r, t, total) if k is not None)
    return got if len(got) > 1 else got[0]


def f8_linear_fwd(x: F8, w: F8, b: torch.Tensor | None = None, act: str = "none", residual: torch.Tensor | None = None,
                  save: str | None = None, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None):
    """y = act(x w^T + b) + residual of packed x (M, I) and w (O, I), in dtype.  save="pre" returns (y, pre) with the
    pre-activation.  In bfloat16 eight products are summed at a time with 13 bits behind the largest's power of two, and those sums
    in float32; in float32 all sums are, which takes up to twice as long.  (So have the gradients'.)"""
    if save not in (None, "pre"):
        raise ValueError(f"save must be None or 'pre', got {save!r}")
    if dtype not in _DT:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    a = _act(act)
    if out is None and type(x) is F8 and type(w) is F8 and x.cols == w.cols:
        made = _train().linear_fwd(x.q, x.e, w.q, w.e, x.cols, b, a, residual, save is not None, _DT[dtype])
        if made is not None:
            return made
    if not isinstance(x, F8):
        raise TypeError(f"x must be packed (pack_f8), got {type(x).__name__}")
    _f8(w, "w", None, x.cols, x.q, second=True)
    M, I, O = x.rows, x.cols, w.rows
    y = torch.empty((M, O), dtype=dtype, device=x.q.device) if out is None else out
    if y.dtype is not dtype:
        raise TypeError(f"out must be {dtype}, got {y.dtype}")
    v, ldy = _same(y, "out", M, O, y)
    if y.get_device() != x.q.get_device():
        raise ValueError(f"out must be on {x.q.device}")
    if b is not None:
        _vector(b, "b", O, y)
    res, ldres = (None, O) if residual is None else _same(residual, "residual", M, O, y)
    pre = torch.empty((M, O), dtype=dtype, device=x.q.device) if save == "pre" else None
    _run("o1d_scaled_linear_fwd", x.q, x.q.data_ptr(), x.e.data_ptr(), _F8_OF[x.q.dtype], w.q.data_ptr(), w.e.data_ptr(),
         None if b is None else b.data_ptr(), a, None if res is None else res.data_ptr(), ldres, v.data_ptr(), ldy,
         None if pre is None else pre.data_ptr(), O, M, I, O, _DT[dtype])
    return y if pre is None else (y, pre)


def f8_linear_bwd_input(dy: F8, wt: F8, pre: torch.Tensor | None = None, act: str = "none",
                        dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None) -> torch.Tensor:
    """dx = (dy w) act'(pre) of packed dy (M, O) and wt, the weights transposed (I, O), in dtype; pre has that type."""
    if dtype not in _DT:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    a = _act(act)
    if (pre is None) != (act == "none"):
        raise ValueError("pre and act are given together")
    if out is None and type(dy) is F8 and type(wt) is F8 and dy.cols == wt.cols:
        made = _train().linear_bwd_input(dy.q, dy.e, wt.q, wt.e, dy.cols, pre, a, _DT[dtype])
        if made is not None:
            return made
    if not isinstance(dy, F8):
        raise TypeError(f"dy must be packed (pack_f8), got {type(dy).__name__}")
    _f8(wt, "wt", None, dy.cols, dy.q, second=True)
    M, O, I = dy.rows, dy.cols, wt.rows
    dx = torch.empty((M, I), dtype=dtype, device=dy.q.device) if out is None else out
    if dx.dtype is not dtype:
        raise TypeError(f"out must be {dtype}, got {dx.dtype}")
    v, lddx = _same(dx, "out", M, I, dx)
    if dx.get_device() != dy.q.get_device():
        raise ValueError(f"out must be on {dy.q.device}")
    p, ldp = (None, I) if pre is None else _same(pre, "pre", M, I, dx)
    _run("o1d_scaled_linear_bwd_input", dy.q, dy.q.data_ptr(), dy.e.data_ptr(), _F8_OF[dy.q.dtype], wt.q.data_ptr(),
         wt.e.data_ptr(), a, None if p is None else p.data_ptr(), ldp, v.data_ptr(), lddx, M, I, O, _DT[dtype])
    return dx


@functools.lru_cache(maxsize=4096)
def f8_linear_workspace_bytes(M: int, I: int, O: int, dtype: torch.dtype) -> int:
    return int(_lib.lib().o1d_scaled_linear_bwd_weight_workspace_bytes(M, I, O, _DT[dtype]))


def f8_linear_bwd_weight(dyt: F8, xt: F8, dtype: torch.dtype = torch.bfloat16, out: torch.Tensor | None = None,
                         workspace: torch.Tensor | None = None) -> torch.Tensor:
    """dw (O, I) = dy^T x of the packed transposes dyt (O, M) and xt (I, M), in dtype."""
    if dtype not in _DT:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    if out is None and workspace is None and type(dyt) is F8 and type(xt) is F8 and dyt.cols == xt.cols:
        dw = _train().linear_bwd_weight(dyt.q, dyt.e, xt.q, xt.e, dyt.cols, _DT[dtype])
        if dw is not None:
            return dw
    if not isinstance(dyt, F8):
        raise TypeError(f"dyt must be packed (pack_f8), got {type(dyt).__name__}")
    _f8(xt, "xt", None, dyt.cols, dyt.q, second=True)
    M, O, I = dyt.cols, dyt.rows, xt.rows
    if O < 1 or I < 1:
        raise ValueError("a weight has at least one row and one column")
    dw = torch.empty((O, I), dtype=dtype, device=dyt.q.device) if out is None else out
    if tuple(dw.shape) != (O, I) or dw.dtype is not dtype or dw.device != dyt.q.device or not dw.is_contiguous():
        raise ValueError(f"out must be a contiguous ({O}, {I}) tensor of {dtype} on {dyt.q.device}")
    workspace, nbytes = _scratch(workspace, dyt.q, f8_linear_workspace_bytes(M, I, O, dtype))
    _run("o1d_scaled_linear_bwd_weight", dyt.q, dyt.q.data_ptr(), dyt.e.data_ptr(), _F8_OF[dyt.q.dtype], xt.q.data_ptr(),
         xt.e.data_ptr(), dw.data_ptr(), M, I, O, _DT[dtype], workspace.data_ptr(), nbytes)
    return dw


class F8LinearFunction(torch.autograd.Function):
    """Autograd glue: y = act(x w^T + b) + residual with products of e4m3 operands; gradients are packed as `grad` ("e5m2"
    or "e4m3").  What the backward needs of x is kept in 8 bits."""

    @staticmethod
    def forward(ctx, x, w, b=None, act="none", residual=None, grad="e5m2"):
        x, w = x.contiguous(), w.contiguous()
        wants = (*ctx.needs_input_grad, False, False, False)  # (arguments left out have no entry)
        xr, xt = pack_f8(x, along="both") if wants[1] and x.numel() else (pack_f8(x), None)
        wr, wt = pack_f8(w, along="both") if wants[0] else (pack_f8(w), None)
        save = None if act == "none" else "pre"
        out = f8_linear_fwd(xr, wr, None if b is None else b.contiguous(), act,
                            None if residual is None else residual.reshape(-1, w.shape[0]).contiguous(), save, x.dtype)
        y, pre = (out, None) if save is None else out
        ctx.act, ctx.grad, ctx.bias, ctx.shape, ctx.dtype = act, grad, b is not None and wants[2], x.shape, x.dtype
        ctx.dtype_w = w.dtype  # (a float32 weight's gradient is not rounded to the input's type)
        ctx.residual = None if residual is None else residual.shape
        ctx.cols = (x.numel() // x.shape[-1], w.shape)
        ctx.save_for_backward(pre, *(k for t in (xt, wt) for k in ((t.q, t.e) if t is not None else (None, None))))
        return y.view(*x.shape[:-1], w.shape[0])

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        pre, xq, xe, wq, we = ctx.saved_tensors
        M, (O, I) = ctx.cols
        wants = (*ctx.needs_input_grad, False, False, False)
        dy = gy.reshape(-1, O).contiguous()
        dh = dy if ctx.act == "none" else act_bwd(pre, dy, ctx.act)
        gx = gw = gb = None
        if wants[0]:
            gx = f8_linear_bwd_input(pack_f8(dh, ctx.grad), F8.of(wq, we, O), dtype=ctx.dtype).view(ctx.shape)
        if wants[1] or ctx.bias:
            if M == 0:
                gw, gb = (dh.new_zeros((O, I), dtype=ctx.dtype_w) if wants[1] else None), (dh.new_zeros((O,)) if ctx.bias else None)
            else:
                dyt, gb = pack_f8(dh, ctx.grad, along="rows", sums=True)
                gb = gb if ctx.bias else None
                gw = f8_linear_bwd_weight(dyt, F8.of(xq, xe, M), dtype=ctx.dtype_w) if wants[1] else None
        return gx, gw, gb, None, (gy.reshape(ctx.residual) if wants[4] else None), None


# ---------------------------------------------------------------- AdamW over many tensors

class AdamState:
    """The states of AdamW for tensors of `sizes` values, flat: tensor i's part starts at `starts[i]`, the sum of the sizes
    before it, each rounded up to 128.  m and v are float32, or float8_e4m3fn (v its root) with float32 scales ms and vs for
    each 128 values; master (or None) the parameters in float32; step int32 (2,), the steps taken and 0 (a negative count is
    read as none)."""

    __slots__ = ("sizes", "starts", "m", "v", "step", "ms", "vs", "master")

    def __init__(self, sizes, m: torch.Tensor, v: torch.Tensor, step: torch.Tensor, ms: torch.Tensor | None = None,
                 vs: torch.Tensor | None = None, master: torch.Tensor | None = None):
        self.sizes = list(sizes)
        self.m, self.v, self.step, self.ms, self.vs, self.master = m, v, step, ms, vs, master
        self.starts = _train().adam_starts(self.sizes, m, v, step, ms, vs, master)
        if self.starts is not None:
            return
        total = sum(-(-n // _lib.SCALED_GROUP) * _lib.SCALED_GROUP for n in self.sizes)
        held8 = m.dtype is torch.float8_e4m3fn
        kinds = [("m", m, (total,), torch.float8_e4m3fn if held8 else torch.float32),
                 ("v", v, (total,), torch.float8_e4m3fn if held8 else torch.float32), ("step", step, (2,), torch.int32)]
        if held8 != (ms is not None) or held8 != (vs is not None):
            raise ValueError("ms and vs are the scales of states in 8 bits, and only of those")
        if held8:
            kinds += [(n, t, (total // _lib.SCALED_GROUP,), torch.float32) for n, t in (("ms", ms), ("vs", vs))]
        if master is not None:
            kinds.append(("master", master, (total,), torch.float32))
        for name, t, shape, dtype in kinds:
            if tuple(t.shape) != shape or t.dtype is not dtype or not t.is_contiguous() or not t.is_cuda \
                    or t.device != m.device:
                raise ValueError(f"{name} must be a contiguous {shape} tensor of {dtype} on one GPU, got {tuple(t.shape)} "
                                 f"{t.dtype} {t.device}")
        raise ValueError(f"no sizes of tensors: {self.sizes}")

    @staticmethod
    def zeros(params, bits: int = 32, master: bool = False) -> "AdamState":
        """New states of these parameters (one device), with master=True their values in float32."""
        params = list(params)
        if bits not in (8, 32) or not params:
            raise ValueError(f"states have 8 or 32 bits, of at least one tensor; got {bits}, {len(params)} tensors")
        device, sizes = params[0].device, [p.numel() for p in params]
        total = sum(-(-n // _lib.SCALED_GROUP) * _lib.SCALED_GROUP for n in sizes)
        kind = torch.float8_e4m3fn if bits == 8 else torch.float32
        m, v = (torch.zeros(total, dtype=torch.uint8 if bits == 8 else kind, device=device).view(kind) for _ in range(2))
        ms, vs = (torch.zeros(total // _lib.SCALED_GROUP, device=device) if bits == 8 else None for _ in range(2))
        flat = torch.zeros(total, device=device) if master else None
        state = AdamState(sizes, m, v, torch.zeros(2, dtype=torch.int32, device=device), ms, vs, flat)
        if master:
            with torch.no_grad():
                for p, n, at in zip(params, sizes, state.starts):
                    flat[at:at + n].copy_(p.reshape(-1))
        return state

    @property
    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in (self.m, self.v, self.ms, self.vs, self.master) if t is not None)


def adamw(params, grads, state: AdamState, lr: float | torch.Tensor = 1e-3, betas: tuple[float, float] = (0.9, 0.999),
          eps: float = 1e-8, weight_decay: float = 0.01, max_norm: float | None = None,
          workspace: torch.Tensor | None = None, follow: bool = False) -> torch.Tensor | None:
    """One AdamW step over all params (of one type, contiguous, each once) in place, as autograd's versions of them tell, given their
    grads (of one type; None leaves a parameter and its states as they are).  lr may be a float32 tensor of one value on the GPU.  max_norm limits the norm of all
    gradients, which is returned; where it is not finite, nothing changes.  With masters the parameters are only written;
    follow=True reads them too, and takes the values of those that are not their masters rounded: somebody wrote them."""
    if max_norm is not None and not max_norm > 0:
        raise ValueError(f"max_norm must be positive, got {max_norm}")
    params, grads = list(params), list(grads)
    if workspace is None:
        made = _train().adamw(params, grads, state.sizes, (state.m, state.v, state.step, state.ms, state.vs, state.master), lr,
                              betas[0], betas[1], eps, weight_decay, max_norm or 0.0, bool(follow))
        if made is not None:
            return None if max_norm is None else made
    if len(params) != len(state.sizes) or len(grads) != len(params):
        raise ValueError(f"{len(params)} parameters and {len(grads)} gradients for the states of {len(state.sizes)}")
    device, pdt, gdt = state.m.device, None, None
    table = (_lib.AdamTensor * max(1, len(params)))()
    count, written = 0, []
    for p, g, n, at in zip(params, grads, state.sizes, state.starts):
        if p.numel() != n or p.device != device or not p.is_contiguous() or (pdt is not None and p.dtype is not pdt):
            raise ValueError(f"parameters must be contiguous tensors of one type on {device} with the states' sizes, got "
                             f"{tuple(p.shape)} {p.dtype} {p.device} for {n} values")
        pdt = p.dtype
        if g is None or n == 0:
            continue
        if g.shape != p.shape or g.device != device or not g.is_contiguous() or (gdt is not None and g.dtype is not gdt):
            raise ValueError(f"gradients must be contiguous tensors of one type with their parameters' shapes, got "
                             f"{tuple(g.shape)} {g.dtype} {g.device} for {tuple(p.shape)}")
        gdt = g.dtype
        table[count] = _lib.AdamTensor(p.data_ptr(), g.data_ptr(), n, at)
        count += 1
        if not p.is_inference():
            written.append(p)
    for t in (pdt, gdt):
        if t is not None and t not in _DT:
            raise TypeError(f"unsupported dtype {t}; use float32 or bfloat16")
    lr_at = None
    if isinstance(lr, torch.Tensor):
        if lr.numel() != 1 or lr.dtype is not torch.float32 or lr.device != device:
            raise ValueError(f"lr must be a number or one float32 value on {device}")
        lr, lr_at = 0.0, lr.data_ptr()
    s = _lib.AdamState(state.m.data_ptr(), state.v.data_ptr(), None if state.ms is None else state.ms.data_ptr(),
                       None if state.vs is None else state.vs.data_ptr(),
                       None if state.master is None else state.master.data_ptr(), state.step.data_ptr(),
                       32 if state.ms is None else 8)
    o = _lib.AdamOptions(lr, betas[0], betas[1], eps, weight_decay, max_norm or 0.0, lr_at, bool(follow))
    norm = state.step.new_empty((), dtype=torch.float32) if max_norm is not None else None
    workspace, nbytes = _scratch(workspace, state.step, int(_lib.lib().o1d_adamw_workspace_bytes(max_norm or 0.0)))
    _run("o1d_adamw", state.step, ctypes.addressof(table), count, _DT[pdt] if pdt else 0, _DT[gdt] if gdt else 0,
         ctypes.addressof(s), ctypes.addressof(o), None if norm is None else norm.data_ptr(), workspace.data_ptr(), nbytes)
    torch.autograd.graph.increment_version(written)
    return norm
