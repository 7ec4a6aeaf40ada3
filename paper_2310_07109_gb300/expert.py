"""ctypes binding of the expert feed-forward operators (include/sparsecoder.h).

Routing of tokens to experts, matrix products grouped by expert and the gated sum
with residual and layer norm, forward and backward.  As in ``binding``: argument
marshalling and checks of types, shapes and devices only, asynchronous on torch's current
stream (or ``stream``), no CPU fallback.  All tensors, the workspace and the stream are
of the current device.  Tokens are the rows of a [B][L] batch with
``rows[b]`` of them in use; slots are (token, choice) pairs in expert order.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import binding as _b

MAX_EXPERTS = 256
MAX_CHOICES = 8
MAX_EXPERT_DIM = 8192

_I, _P, _F, _LL = ctypes.c_int, ctypes.c_void_p, ctypes.c_float, ctypes.c_longlong


class RouteArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("L", _I), ("E", _I), ("k", _I), ("logits", _P), ("ld", _LL),
                ("rows", _P), ("renormalize", _I), ("expert", _P), ("gate", _P),
                ("offsets", _P), ("slot", _P), ("token", _P)]


class RouteBackwardArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("L", _I), ("E", _I), ("k", _I), ("logits", _P), ("ld", _LL),
                ("rows", _P), ("renormalize", _I), ("expert", _P), ("gate", _P),
                ("dgate", _P), ("dlogits", _P)]


class ExpertLinearArgs(ctypes.Structure):
    _fields_ = [("M", _I), ("E", _I), ("N", _I), ("K", _I), ("X", _P), ("ldx", _LL),
                ("x_rows", _I), ("token", _P), ("offsets", _P), ("W", _P), ("bias", _P),
                ("gelu", _I), ("pre", _P), ("out", _P), ("out_f32", _I)]


class ExpertLinearBackwardInputArgs(ctypes.Structure):
    _fields_ = [("M", _I), ("E", _I), ("N", _I), ("K", _I), ("dY", _P), ("ldy", _LL),
                ("offsets", _P), ("W", _P), ("pre", _P), ("dX", _P), ("out_f32", _I)]


class ExpertLinearBackwardWeightArgs(ctypes.Structure):
    _fields_ = [("M", _I), ("E", _I), ("N", _I), ("K", _I), ("dY", _P), ("ldy", _LL), ("X", _P),
                ("ldx", _LL), ("x_rows", _I), ("token", _P), ("offsets", _P), ("dW", _P),
                ("out_f32", _I), ("dbias", _P)]


class ExpertCombineArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("L", _I), ("D", _I), ("k", _I), ("M", _I), ("rows", _P), ("Y", _P),
                ("slot", _P), ("gate", _P), ("res", _P), ("res_scale", _F), ("gamma", _P),
                ("beta", _P), ("eps", _F), ("sum", _P), ("out", _P)]


class ExpertCombineBackwardArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("L", _I), ("D", _I), ("k", _I), ("M", _I), ("rows", _P), ("Y", _P),
                ("slot", _P), ("gate", _P), ("res", _P), ("res_scale", _F), ("gamma", _P),
                ("eps", _F), ("dout", _P), ("dsum", _P), ("dY", _P), ("dgate", _P), ("dres", _P),
                ("dgamma", _P), ("dbeta", _P)]


# calls with a workspace and its size before the stream, and those without
_WITH_WORKSPACE = {"sc_expert_route_forward": RouteArgs,
                   "sc_expert_linear_forward": ExpertLinearArgs,
                   "sc_expert_linear_backward_input": ExpertLinearBackwardInputArgs,
                   "sc_expert_linear_backward_weight": ExpertLinearBackwardWeightArgs,
                   "sc_expert_combine_backward": ExpertCombineBackwardArgs}
_WITHOUT_WORKSPACE = {"sc_expert_route_backward": RouteBackwardArgs,
                      "sc_expert_combine_forward": ExpertCombineArgs}
_bound = None


def _library():
    global _bound
    if _bound is None:
        lib = _b.load()
        for name, args in _WITH_WORKSPACE.items():
            getattr(lib, name).argtypes = [ctypes.POINTER(args), _P, ctypes.c_size_t, _P]
        for name, args in _WITHOUT_WORKSPACE.items():
            getattr(lib, name).argtypes = [ctypes.POINTER(args), _P]
        lib.sc_expert_workspace_size.restype = ctypes.c_size_t
        lib.sc_expert_workspace_size.argtypes = [_I] * 5
        _bound = lib
    return _bound


class _Entry:
    """An entry point called with its argument block packed by ``struct``: a call on a few
    rows is all launch time, and filling in a ctypes structure takes a tenth of that."""

    def __init__(self, name):
        self.name, self.call = name, None
        args = _WITH_WORKSPACE.get(name) or _WITHOUT_WORKSPACE[name]
        code = {_I: "i", _P: "P", _F: "f", _LL: "q"}
        self.pack = struct.Struct("@" + "".join(code[t] for _, t in args._fields_)).pack

    def bind(self):
        rest = [_P, ctypes.c_size_t, _P] if self.name in _WITH_WORKSPACE else [_P]
        self.call = ctypes.CFUNCTYPE(_I, ctypes.c_char_p, *rest)((self.name, _library()))
        return self.call


_ROUTE, _ROUTE_BACK = _Entry("sc_expert_route_forward"), _Entry("sc_expert_route_backward")
_LINEAR, _COMBINE = _Entry("sc_expert_linear_forward"), _Entry("sc_expert_combine_forward")
_BACK_X, _BACK_W = _Entry("sc_expert_linear_backward_input"), _Entry("sc_expert_linear_backward_weight")
_COMBINE_BACK = _Entry("sc_expert_combine_backward")


def _refuse(what):
    raise _b.SparseCoderError(_b.SC_ERR_INVALID_ARG, what)


# The library launches on the current device (torch.cuda.current_device() first checks that
# CUDA is set up, which a call with cuda tensors need not).
_current_device = getattr(torch._C, "_cuda_getDevice", None)


def _device(t, name):
    """The device of a call's first tensor: the current one, which the library launches on.
    (A stream's raw handle and pointers of another device would be used on this one.)"""
    dev = t.get_device()
    if dev < 0:
        _refuse("%s: a cuda tensor is wanted" % name)
    if dev != _current_device():
        _refuse("%s is on cuda:%d, the current device is cuda:%d" % (name, dev, _current_device()))
    return dev


def _at(t, name, dtype, count, dev):
    """The address of a contiguous tensor of this type on this device with so many elements
    (their shape may be any that the rows run through in order); 0 for None."""
    if t is None:
        return 0
    if t.dtype is dtype and t.numel() == count and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    _refuse("%s: a contiguous tensor of %s on cuda:%d with %d elements is wanted" % (name, dtype, dev, count))


def _rows_at(t, name, dtype, dev):
    """Address, rows, width and row distance of a matrix whose rows are contiguous."""
    if t.dim() != 2 or t.dtype is not dtype or t.get_device() != dev:
        _refuse("%s: a matrix of %s on cuda:%d is wanted" % (name, dtype, dev))
    rows, width = t.shape
    ld, step = t.stride()
    if step != 1 and width > 1:
        _refuse("%s: contiguous rows are wanted" % name)
    return t.data_ptr(), rows, width, ld if rows > 1 else max(ld, width)


def _stream(stream, dev):
    # the raw handle: torch.cuda.current_stream() takes as long as a small kernel
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        _refuse("the stream is of cuda:%d, the tensors are on cuda:%d" % (stream.device_index, dev))
    return stream.cuda_stream


def _shape(t, name, dims):
    """The shape of a tensor of so many dimensions."""
    if t.dim() != dims:
        _refuse("%s: %d dimensions are wanted" % (name, dims))
    return t.shape


def _made(stream, *tensors):
    """Outputs made on the current stream for a call on ``stream``."""
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream(tensors[0].device))   # what had the memory before
        for t in tensors:
            t.record_stream(stream)


def _out_type(t):
    if t.dtype is torch.float32:
        return 1
    if t.dtype is torch.bfloat16:
        return 0
    _refuse("outputs are bfloat16 or float32")


def expert_workspace_size(B, L, E, k, D) -> int:
    return int(_library().sc_expert_workspace_size(int(B), int(L), int(E), int(k), int(D)))


def new_expert_workspace(B, L, E, k, D, device=None) -> torch.Tensor:
    """Workspace of the expert operators for a [B][L] batch, E experts, k choices and rows
    of at most D features (zeroed, 256-byte aligned)."""
    n = expert_workspace_size(B, L, E, k, D)
    if n == 0:
        raise _b.SparseCoderError(_b.SC_ERR_INVALID_ARG, "invalid expert workspace sizes")
    ws = torch.zeros(n + 256, dtype=torch.uint8, device=device or "cuda")
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n]


def _work(workspace, device, stream, B, L, E, k, D):
    if workspace is not None:
        return workspace
    ws = new_expert_workspace(B, L, E, k, D, device)
    if stream is not None:
        # made (and zeroed) on the current stream, used and let go on another
        stream.wait_stream(torch.cuda.current_stream(device))
        ws.record_stream(stream)
    return ws


def _call(entry, args, ws, dev, stream):
    if ws.get_device() != dev:
        _refuse("workspace: a tensor on cuda:%d is wanted" % dev)
    rc = (entry.call or entry.bind())(args, ws.data_ptr(), ws.numel(), _stream(stream, dev))
    if rc:
        _b._check(rc)


def _call_plain(entry, args, dev, stream):
    rc = (entry.call or entry.bind())(args, _stream(stream, dev))
    if rc:
        _b._check(rc)


def expert_route_forward(logits, *, k, B, L, rows=None, renormalize=True, out=None, workspace=None,
                         stream=None):
    """``sc_expert_route_forward``: logits fp32 [B*L, E] (any row stride) to k experts a token.
    Returns dict(expert [B*L, k] int32, gate [B*L, k] fp32, offsets [E + 1], slot [B*L, k],
    token [B*L*k] int32)."""
    dev = _device(logits, "logits")
    at, T, E, ld = _rows_at(logits, "logits", torch.float32, dev)
    if T != B * L:
        _refuse("logits: B * L rows are wanted")
    if out is None:
        new = lambda *shape, dtype=torch.int32: torch.empty(shape, dtype=dtype, device=logits.device)  # noqa: E731
        out = {"expert": new(T, k), "gate": new(T, k, dtype=torch.float32), "offsets": new(E + 1),
               "slot": new(T, k), "token": new(T * k)}
        _made(stream, *out.values())
    i32 = torch.int32
    a = _ROUTE.pack(B, L, E, k, at, ld, _at(rows, "rows", i32, B, dev), 1 if renormalize else 0,
                  _at(out["expert"], "expert", i32, T * k, dev),
                  _at(out["gate"], "gate", torch.float32, T * k, dev),
                  _at(out["offsets"], "offsets", i32, E + 1, dev),
                  _at(out["slot"], "slot", i32, T * k, dev), _at(out["token"], "token", i32, T * k, dev))
    _call(_ROUTE, a, _work(workspace, logits.device, stream, B, L, E, k, 8), dev, stream)
    return out


def expert_route_backward(logits, expert, gate, dgate, *, B, L, rows=None, renormalize=True, out=None,
                          stream=None):
    """``sc_expert_route_backward``: the gradient of the logits, fp32 [B*L, E]."""
    dev = _device(logits, "logits")
    at, T, E, ld = _rows_at(logits, "logits", torch.float32, dev)
    if T != B * L:
        _refuse("logits: B * L rows are wanted")
    k = _shape(expert, "expert", 2)[1]
    if out is None:
        out = torch.empty((T, E), dtype=torch.float32, device=logits.device)
        _made(stream, out)
    f32 = torch.float32
    a = _ROUTE_BACK.pack(B, L, E, k, at, ld, _at(rows, "rows", torch.int32, B, dev),
                          1 if renormalize else 0, _at(expert, "expert", torch.int32, T * k, dev),
                          _at(gate, "gate", f32, T * k, dev), _at(dgate, "dgate", f32, T * k, dev),
                          _at(out, "dlogits", f32, T * E, dev))
    _call_plain(_ROUTE_BACK, a, dev, stream)
    return out


# Per device: the workspace of products that are called without one.  They use its status
# word alone, which only ever gains bits, so that calls on several streams may share it.
_products = {}


def _product_ws(workspace, t, dev, stream):
    if workspace is not None:
        return workspace
    ws = _products.get(dev)
    if ws is None:
        if torch.cuda.is_current_stream_capturing():
            return _work(None, t.device, stream, 1, 1, 1, 1, 8)   # a graph's memory is not kept
        ws = new_expert_workspace(1, 1, 1, 1, 8, t.device)
        torch.cuda.current_stream(t.device).synchronize()   # zeroed, for whatever stream comes first
        ws = _products.setdefault(dev, ws)
    return ws


def expert_status(stream=None) -> int:
    """Synchronise ``stream`` (the current one) and return, then clear, the status of the products
    called without a workspace on the current device, outside a graph capture.  A workspace's
    own status: ``workspace_status``."""
    ws = _products.get(torch.cuda.current_device())
    return _b.SC_OK if ws is None else _b.workspace_status(ws, stream)


def expert_linear_forward(X, W, offsets, *, token=None, bias=None, gelu=False, pre=None, out=None,
                          out_f32=False, workspace=None, stream=None):
    """``sc_expert_linear_forward``: X bf16 [rows, K] (any row stride), W bf16 [E, N, K], offsets
    int32 [E + 1], bias fp32 [E, N].  Slot s reads row token[s] of X, or row s.  ``pre``: a
    bf16 [M, N] tensor that receives the values before GELU.  Returns out [M, N], M = len(token),
    or the rows of X."""
    dev = _device(X, "X")
    at, xr, K, ld = _rows_at(X, "X", torch.bfloat16, dev)
    E, N, _ = _shape(W, "W", 3)
    M = xr if token is None else token.numel()
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32 if out_f32 else torch.bfloat16, device=X.device)
        _made(stream, out)
    i32 = torch.int32
    a = _LINEAR.pack(M, E, N, K, at, ld, xr, _at(token, "token", i32, M, dev),
                         _at(offsets, "offsets", i32, E + 1, dev), _at(W, "W", torch.bfloat16, E * N * K, dev),
                         _at(bias, "bias", torch.float32, E * N, dev), 1 if gelu else 0,
                         _at(pre, "pre", torch.bfloat16, M * N, dev), _at(out, "out", out.dtype, M * N, dev),
                         _out_type(out))
    _call(_LINEAR, a, _product_ws(workspace, X, dev, stream), dev, stream)
    return out


def expert_linear_backward_input(dY, W, offsets, *, pre=None, out=None, out_f32=False, workspace=None,
                                 stream=None):
    """``sc_expert_linear_backward_input``: dY bf16 [M, N] (any row stride), W bf16 [E, N, K]; with
    ``pre`` bf16 [M, K] the result is multiplied by GELU'(pre).  Returns dX [M, K]."""
    dev = _device(dY, "dY")
    at, M, N, ld = _rows_at(dY, "dY", torch.bfloat16, dev)
    E, _, K = _shape(W, "W", 3)
    if out is None:
        out = torch.empty((M, K), dtype=torch.float32 if out_f32 else torch.bfloat16, device=dY.device)
        _made(stream, out)
    a = _BACK_X.pack(M, E, N, K, at, ld, _at(offsets, "offsets", torch.int32, E + 1, dev),
                                      _at(W, "W", torch.bfloat16, E * N * K, dev),
                                      _at(pre, "pre", torch.bfloat16, M * K, dev),
                                      _at(out, "out", out.dtype, M * K, dev), _out_type(out))
    _call(_BACK_X, a, _product_ws(workspace, dY, dev, stream), dev, stream)
    return out


def expert_linear_backward_weight(dY, X, offsets, *, token=None, bias=True, out=None, out_f32=True,
                                  workspace=None, stream=None):
    """``sc_expert_linear_backward_weight``: dY bf16 [M, N], X bf16 [rows, K] (any row strides).
    Returns dict(dW [E, N, K], dbias fp32 [E, N]); without dbias when ``bias`` is False (or
    ``out`` has none)."""
    dev = _device(dY, "dY")
    ay, M, N, ldy = _rows_at(dY, "dY", torch.bfloat16, dev)
    ax, xr, K, ldx = _rows_at(X, "X", torch.bfloat16, dev)
    E = _shape(offsets, "offsets", 1)[0] - 1
    if out is None:
        out = {"dW": torch.empty((E, N, K), dtype=torch.float32 if out_f32 else torch.bfloat16,
                                 device=X.device)}
        if bias:
            out["dbias"] = torch.empty((E, N), dtype=torch.float32, device=X.device)
        _made(stream, *out.values())
    dW = out["dW"]
    a = _BACK_W.pack(M, E, N, K, ay, ldy, ax, ldx, xr,
                                       _at(token, "token", torch.int32, M, dev),
                                       _at(offsets, "offsets", torch.int32, E + 1, dev),
                                       _at(dW, "dW", dW.dtype, E * N * K, dev), _out_type(dW),
                                       _at(out.get("dbias"), "dbias", torch.float32, E * N, dev))
    _call(_BACK_W, a, _product_ws(workspace, X, dev, stream), dev, stream)
    return out


def expert_combine_forward(Y, slot, gate=None, *, B, L, rows=None, res=None, res_scale=1.0, gamma=None,
                           beta=None, eps=1e-5, out=None, stream=None):
    """``sc_expert_combine_forward``: Y bf16 [M, D] rows of the slots, slot int32 [B*L, k], gate fp32
    [B*L, k] or None (1), res bf16 [B*L, D].  Returns dict(sum [B*L, D] bf16, out) (``out`` with
    gamma and beta only); a given ``out`` may lack "sum" where there is a norm."""
    dev = _device(Y, "Y")
    M, D = _shape(Y, "Y", 2)
    T, k = B * L, _shape(slot, "slot", 2)[1]
    if out is None:
        out = {"sum": torch.empty((T, D), dtype=torch.bfloat16, device=Y.device)}
        if gamma is not None:
            out["out"] = torch.empty((T, D), dtype=torch.bfloat16, device=Y.device)
        _made(stream, *out.values())
    bf, f32 = torch.bfloat16, torch.float32
    a = _COMBINE.pack(B, L, D, k, M, _at(rows, "rows", torch.int32, B, dev), _at(Y, "Y", bf, M * D, dev),
                          _at(slot, "slot", torch.int32, T * k, dev), _at(gate, "gate", f32, T * k, dev),
                          _at(res, "res", bf, T * D, dev), res_scale, _at(gamma, "gamma", f32, D, dev),
                          _at(beta, "beta", f32, D, dev), eps, _at(out.get("sum"), "sum", bf, T * D, dev),
                          _at(out.get("out"), "out", bf, T * D, dev))
    _call_plain(_COMBINE, a, dev, stream)
    return out


def expert_combine_backward(Y, slot, gate=None, *, B, L, dout=None, dsum=None, rows=None, res=None,
                            res_scale=1.0, gamma=None, eps=1e-5, out=None, workspace=None, stream=None):
    """``sc_expert_combine_backward``: gradients from dout (with gamma) and dsum, bf16 [B*L, D].
    Returns dict(dY [M, D] bf16, dgate [B*L, k] fp32, dres [B*L, D] bf16 where res is given, dgamma
    and dbeta [D] fp32 where gamma is)."""
    dev = _device(Y, "Y")
    M, D = _shape(Y, "Y", 2)
    T, k = B * L, _shape(slot, "slot", 2)[1]
    bf, f32 = torch.bfloat16, torch.float32
    if out is None:
        new = lambda *shape, dtype=f32: torch.empty(shape, dtype=dtype, device=Y.device)  # noqa: E731
        out = {"dY": new(M, D, dtype=bf), "dgate": new(T, k)}
        if res is not None:
            out["dres"] = new(T, D, dtype=bf)
        if gamma is not None:
            out.update(dgamma=new(D), dbeta=new(D))
        _made(stream, *out.values())
    a = _COMBINE_BACK.pack(
        B, L, D, k, M, _at(rows, "rows", torch.int32, B, dev), _at(Y, "Y", bf, M * D, dev),
        _at(slot, "slot", torch.int32, T * k, dev), _at(gate, "gate", f32, T * k, dev),
        _at(res, "res", bf, T * D, dev), res_scale, _at(gamma, "gamma", f32, D, dev), eps,
        _at(dout, "dout", bf, T * D, dev), _at(dsum, "dsum", bf, T * D, dev), _at(out["dY"], "dY", bf, M * D, dev),
        _at(out.get("dgate"), "dgate", f32, T * k, dev), _at(out.get("dres"), "dres", bf, T * D, dev),
        _at(out.get("dgamma"), "dgamma", f32, D, dev), _at(out.get("dbeta"), "dbeta", f32, D, dev))
    _call(_COMBINE_BACK, a, _work(workspace, Y.device, stream, B, L, 1, 1, D), dev, stream)
    return out
