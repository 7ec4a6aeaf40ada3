"""ctypes binding of the pruned key-value cache (include/sparsecoder.h).

Norm and rotation of query and key heads, forward and backward, and the incremental form of the
framework's attention with token pruning: keys and values appended to a cache, attention
over it with the weights added up for each slot, eviction of the slots with the least.  As in
``binding`` and ``expert``: argument marshalling and checks of types, shapes and devices only,
asynchronous on torch's current stream (or ``stream``), no CPU fallback.  All tensors, the
workspace and the stream are of the current device.

Tokens are the rows of a [B][L] batch with ``rows[b]`` of them in use.  A cache is a dict of
tensors (``new_cache``): K, V [B, Hk, C, d] of bfloat16 or float16 (any strides that are multiples of 8; d
contiguous), acc fp32 and pos int32 [B, lists, C], len int32 [B, lists], seen int32 [B].  Its calls
change it in place; ``out`` may name other tensors for what they replace, and for any of the new ones.
"""
from __future__ import annotations

import ctypes
import math
import struct

import torch

from . import binding as _b
from .expert import _at, _device, _made, _refuse, _stream

MAX_HEAD_WIDTH = 256
MAX_HEADS = 1024
MAX_CACHE = 262144
MAX_STEP = 4096

_I, _P, _F, _LL = ctypes.c_int, ctypes.c_void_p, ctypes.c_float, ctypes.c_longlong
_TURN = [("eps", _F), ("rot", _I), ("interleaved", _I), ("freq", _P), ("mscale", _F)]
_CACHE = [("d", _I), ("dtype", _I), ("K", _P), ("V", _P), ("stride_b", _LL), ("stride_h", _LL), ("stride_c", _LL),
          ("acc", _P), ("pos", _P), ("len", _P), ("seen", _P)]


class RotateArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("L", _I), ("Hq", _I), ("Hk", _I), ("d", _I), ("dtype", _I), ("Q", _P), ("ldq", _LL),
                ("K", _P), ("ldk", _LL), ("rows", _P), ("pos", _P), ("gamma_q", _P), ("gamma_k", _P), *_TURN,
                ("Q_out", _P), ("ldq_out", _LL), ("K_out", _P), ("ldk_out", _LL)]


class RotateBackwardArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("L", _I), ("Hq", _I), ("Hk", _I), ("d", _I), ("dtype", _I), ("dQ_out", _P), ("ldq_out", _LL),
                ("dK_out", _P), ("ldk_out", _LL), ("Q", _P), ("ldq", _LL), ("K", _P), ("ldk", _LL), ("rows", _P), ("pos", _P),
                ("gamma_q", _P), ("gamma_k", _P), *_TURN, ("dQ", _P), ("ldq_grad", _LL), ("dK", _P), ("ldk_grad", _LL),
                ("dgamma_q", _P), ("dgamma_k", _P)]


class CacheAppendArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("C", _I), ("H", _I), ("Hk", _I), ("G", _I), *_CACHE, ("L", _I), ("Q", _P), ("ldq", _LL),
                ("K_in", _P), ("ldk", _LL), ("V_in", _P), ("ldv", _LL), ("rows", _P), ("gamma_q", _P), ("gamma_k", _P), *_TURN,
                ("Q_out", _P), ("ldq_out", _LL), ("len_out", _P), ("seen_out", _P)]


class CacheAttendArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("C", _I), ("H", _I), ("Hk", _I), ("G", _I), *_CACHE, ("T", _I), ("Q", _P), ("ldq", _LL),
                ("rows", _P), ("scale", _F), ("decay", _F), ("O", _P), ("ldo", _LL), ("acc_out", _P)]


class CacheEvictArgs(ctypes.Structure):
    _fields_ = [("B", _I), ("C", _I), ("Hk", _I), ("G", _I), *_CACHE, ("budget", _I), ("slack", _I), ("sinks", _I),
                ("recent", _I), ("acc_out", _P), ("pos_out", _P), ("len_out", _P)]


_bound = None


def _library():
    global _bound
    if _bound is None:
        lib = _b.load()
        for entry in (_ROTATE_BACK, _APPEND, _ATTEND, _EVICT):
            getattr(lib, entry.name).argtypes = [ctypes.POINTER(entry.args), _P, ctypes.c_size_t, _P]
        lib.sc_rotate_forward.argtypes = [ctypes.POINTER(RotateArgs), _P]
        lib.sc_rotate_workspace_size.restype = lib.sc_cache_workspace_size.restype = ctypes.c_size_t
        lib.sc_rotate_workspace_size.argtypes = [_I]
        lib.sc_cache_workspace_size.argtypes = [_I] * 7
        _bound = lib
    return _bound


class _Entry:
    """An entry point called with its argument block packed by ``struct``: a step on one
    token is all launch time."""

    def __init__(self, name, args, workspace=True):
        self.name, self.args, self.workspace, self.call = name, args, workspace, None
        code = {_I: "i", _P: "P", _F: "f", _LL: "q"}
        self.pack = struct.Struct("@" + "".join(code[t] for _, t in args._fields_)).pack

    def bind(self):
        rest = [_P, ctypes.c_size_t, _P] if self.workspace else [_P]
        self.call = ctypes.CFUNCTYPE(_I, ctypes.c_char_p, *rest)((self.name, _library()))
        return self.call


_ROTATE = _Entry("sc_rotate_forward", RotateArgs, workspace=False)
_ROTATE_BACK = _Entry("sc_rotate_backward", RotateBackwardArgs)
_APPEND = _Entry("sc_cache_append", CacheAppendArgs)
_ATTEND = _Entry("sc_cache_attend", CacheAttendArgs)
_EVICT = _Entry("sc_cache_evict", CacheEvictArgs)


def _call(entry, args, ws, dev, stream):
    if ws.get_device() != dev:
        _refuse("workspace: a tensor on cuda:%d is wanted" % dev)
    rc = (entry.call or entry.bind())(args, ws.data_ptr(), ws.numel(), _stream(stream, dev))
    if rc:
        _b._check(rc)


def _aligned(n, device):
    if n == 0:
        raise _b.SparseCoderError(_b.SC_ERR_INVALID_ARG, "invalid workspace sizes")
    ws = torch.zeros(n + 256, dtype=torch.uint8, device=device or "cuda")
    off = (-ws.data_ptr()) % 256
    return ws[off:off + n]


def _own_work(ws, device, stream):
    """A workspace made (and zeroed) on the current stream for one call on ``stream``."""
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream(device))
        ws.record_stream(stream)
    return ws


def rotate_workspace_size(width) -> int:
    return int(_library().sc_rotate_workspace_size(int(width)))


def new_rotate_workspace(width, device=None) -> torch.Tensor:
    """Workspace of ``rotate_backward`` for heads of ``width`` features (zeroed, 256-byte aligned)."""
    return _aligned(rotate_workspace_size(width), device)


def cache_workspace_size(B, C, H, heads, *, width=64, lists=1, T=1) -> int:
    return int(_library().sc_cache_workspace_size(int(B), int(C), int(H), int(heads), int(lists), int(width), int(T)))


def new_cache_workspace(B, C, H, heads, *, width=64, lists=1, T=1, device=None) -> torch.Tensor:
    """Workspace of the cache's calls: H query heads, ``heads`` key heads, at most T tokens a
    sequence in one ``cache_attend`` (zeroed, 256-byte aligned)."""
    return _aligned(cache_workspace_size(B, C, H, heads, width=width, lists=lists, T=T), device)


def new_cache(B, C, heads, *, width=64, lists=1, dtype=torch.bfloat16, device=None) -> dict:
    """An empty cache of C slots a list; ``lists`` divides ``heads``."""
    dev = device or "cuda"
    zeros = lambda *shape, dtype: torch.zeros(shape, dtype=dtype, device=dev)  # noqa: E731
    i32 = torch.int32
    return {"K": zeros(B, heads, C, width, dtype=dtype), "V": zeros(B, heads, C, width, dtype=dtype),
            "acc": zeros(B, lists, C, dtype=torch.float32), "pos": zeros(B, lists, C, dtype=i32),
            "len": zeros(B, lists, dtype=i32), "seen": zeros(B, dtype=i32)}


def rotary_frequencies(rot, base=10000.0, *, method=None, factor=1.0, length=0, low=1.0, high=32.0, device=None):
    """(freq, mscale) for ``rot`` rotated features: f_i = base^(-2 i / rot) radians a position, and
    for contexts ``factor`` times as long as a model was trained on:
      "linear"  f / factor
      "base"    base factor^(rot / (rot - 2)) in place of base: the lowest frequency becomes f / factor, the highest stays
      "parts"   by the turns t = length f / (2 pi) that a pair makes over the trained ``length``: f above ``high`` turns,
                f / factor below ``low``, in between linear in t; mscale = 0.1 ln(factor) + 1
    freq is a float64 tensor."""
    if method not in (None, "linear", "base", "parts") or rot < 2 or rot % 2 or not factor >= 1.0 or (
            method == "base" and rot == 2) or (method == "parts" and not (length > 0 and high > low)):
        _refuse("rotary_frequencies: rot is even, factor at least 1, method None, linear, base or parts (with a length, low < high)")
    if method == "base":
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if method == "linear":
        f = [x / factor for x in f]
    elif method == "parts":
        part = [min(max((length * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [x * (g + (1 - g) / factor) for x, g in zip(f, part)]
    return torch.tensor(f, dtype=torch.float64, device=device or "cuda"), 0.1 * math.log(factor) + 1 if method == "parts" else 1.0


_TYPES = {torch.bfloat16: 0, torch.float16: 1}


def _type(t):
    code = _TYPES.get(t.dtype)
    if code is None:
        _refuse("tensors of bfloat16 or float16 are wanted")
    return code


def _heads_at(t, name, dtype, T, d, dev):
    """Address, heads and token distance of a matrix [T, heads * d]; none for None."""
    if t is None:
        return 0, 0, 0
    shape = t.shape
    if len(shape) == 2 and t.dtype is dtype and t.get_device() == dev and shape[0] == T and shape[1] % d == 0:
        ld, step = t.stride()
        if step == 1 or shape[1] == 1:
            return t.data_ptr(), shape[1] // d, ld if T > 1 else shape[1]
    _refuse("%s: %d rows of heads of %d features, of %s on cuda:%d and contiguous, are wanted" % (name, T, d, dtype, dev))


def _turn_at(freq, gamma_q, gamma_k, d, dev):
    f32 = torch.float32
    rot = 0 if freq is None else 2 * freq.numel()
    return _at(gamma_q, "gamma_q", f32, d, dev), _at(gamma_k, "gamma_k", f32, d, dev), rot, \
        _at(freq, "freq", torch.float64, rot // 2, dev)


def _same(a, b, what):
    if a != b:
        _refuse("%s: as many heads as of the input are wanted" % what)


def _rest(out, wanted, device, stream):
    """``out`` and a new tensor for each output that it does not name; wanted: name, shape, type."""
    made = {n: torch.empty(shape, dtype=dt, device=device) for n, shape, dt in wanted if out is None or n not in out}
    if made:
        _made(stream, *made.values())
    return {**(out or {}), **made} if made or out is None else out


def rotate_forward(Q, K=None, *, width, B, L, rows=None, pos=None, freq=None, interleaved=False, mscale=1.0, gamma_q=None,
                   gamma_k=None, eps=1e-6, out=None, stream=None):
    """``sc_rotate_forward``: Q [B*L, Hq * width], K [B*L, Hk * width] (row strides multiples of 8; one may be None),
    pos int32 [B, L] (None: the row), freq float64 [rot / 2] (None: no rotation).  Returns dict(Q, K) of what was given."""
    first = Q if Q is not None else K
    if first is None:
        _refuse("Q or K is wanted")
    dev, dt, code = _device(first, "Q"), first.dtype, _type(first)
    if width < 1:
        _refuse("width: at least 1 is wanted")
    q, Hq, ldq = _heads_at(Q, "Q", dt, B * L, width, dev)
    k, Hk, ldk = _heads_at(K, "K", dt, B * L, width, dev)
    out = _rest(out, [(n, (B * L, h * width), dt) for n, h in (("Q", Hq), ("K", Hk)) if h], first.device, stream)
    qo, hq, ldqo = _heads_at(out["Q"] if Hq else None, "out Q", dt, B * L, width, dev)
    ko, hk, ldko = _heads_at(out["K"] if Hk else None, "out K", dt, B * L, width, dev)
    _same(hq, Hq, "out Q")
    _same(hk, Hk, "out K")
    gq, gk, rot, f = _turn_at(freq, gamma_q, gamma_k, width, dev)
    a = _ROTATE.pack(B, L, Hq, Hk, width, code, q, ldq, k, ldk, _at(rows, "rows", torch.int32, B, dev),
                     _at(pos, "pos", torch.int32, B * L, dev), gq, gk, eps, rot, 1 if interleaved else 0, f, mscale,
                     qo, ldqo, ko, ldko)
    rc = (_ROTATE.call or _ROTATE.bind())(a, _stream(stream, dev))
    if rc:
        _b._check(rc)
    return out


def rotate_backward(dQ, dK=None, Q=None, K=None, *, width, B, L, rows=None, pos=None, freq=None, interleaved=False, mscale=1.0,
                    gamma_q=None, gamma_k=None, eps=1e-6, out=None, workspace=None, stream=None):
    """``sc_rotate_backward``: gradients from dQ [B*L, Hq * width] and dK, of the outputs; Q, K, the forward
    call's inputs, where there is a norm.  Returns dict(dQ, dK, and dgamma_q, dgamma_k [width] fp32 where gamma is given)."""
    first = dQ if dQ is not None else dK
    if first is None:
        _refuse("dQ or dK is wanted")
    dev, dt, code = _device(first, "dQ"), first.dtype, _type(first)
    if width < 1:
        _refuse("width: at least 1 is wanted")
    dq, Hq, ldqo = _heads_at(dQ, "dQ", dt, B * L, width, dev)
    dk, Hk, ldko = _heads_at(dK, "dK", dt, B * L, width, dev)
    q, hq, ldq = _heads_at(Q if gamma_q is not None and Hq else None, "Q", dt, B * L, width, dev)
    k, hk, ldk = _heads_at(K if gamma_k is not None and Hk else None, "K", dt, B * L, width, dev)
    if (gamma_q is not None and hq != Hq) or (gamma_k is not None and hk != Hk):
        _refuse("Q, K: the forward call's inputs are wanted where there is a norm")
    wanted = [(n, (B * L, h * width), dt) for n, h in (("dQ", Hq), ("dK", Hk)) if h]
    wanted += [(n, (width,), torch.float32) for n, gamma in (("dgamma_q", gamma_q), ("dgamma_k", gamma_k)) if gamma is not None]
    out = _rest(out, wanted, first.device, stream)
    qg, hq, ldqg = _heads_at(out["dQ"] if Hq else None, "out dQ", dt, B * L, width, dev)
    kg, hk, ldkg = _heads_at(out["dK"] if Hk else None, "out dK", dt, B * L, width, dev)
    _same(hq, Hq, "out dQ")
    _same(hk, Hk, "out dK")
    gq, gk, rot, f = _turn_at(freq, gamma_q, gamma_k, width, dev)
    f32 = torch.float32
    a = _ROTATE_BACK.pack(B, L, Hq, Hk, width, code, dq, ldqo, dk, ldko, q, ldq, k, ldk, _at(rows, "rows", torch.int32, B, dev),
                          _at(pos, "pos", torch.int32, B * L, dev), gq, gk, eps, rot, 1 if interleaved else 0, f, mscale,
                          qg, ldqg, kg, ldkg, _at(out["dgamma_q"] if gq else None, "dgamma_q", f32, width, dev),
                          _at(out["dgamma_k"] if gk else None, "dgamma_k", f32, width, dev))
    ws = workspace if workspace is not None else _own_work(new_rotate_workspace(width, first.device), first.device, stream)
    _call(_ROTATE_BACK, a, ws, dev, stream)
    return out


def _cache_at(cache, dev):
    """(B, Hk, C, G, d, dtype of torch), and the argument block's part on the cache."""
    K, V, acc, pos, length, seen = cache["K"], cache["V"], cache["acc"], cache["pos"], cache["len"], cache["seen"]
    shape, strides, dt = K.shape, K.stride(), K.dtype
    if len(shape) != 4 or V.shape != shape or V.dtype is not dt or K.get_device() != dev or V.get_device() != dev:
        _refuse("K, V: two tensors [B, heads, C, d] of one type on cuda:%d are wanted" % dev)
    if V.stride() != strides or (strides[3] != 1 and shape[3] > 1):
        _refuse("K, V: the same strides, with contiguous features, are wanted")
    B, Hk, C, d = shape
    lists = length.shape
    if len(lists) != 2 or lists[0] != B:
        _refuse("len: [B, lists] is wanted")
    G, i32 = lists[1], torch.int32
    sb, sh, sc, _ = strides
    return (B, Hk, C, G, d, dt), (
        d, _type(K), K.data_ptr(), V.data_ptr(), sb if B > 1 else 0, sh if Hk > 1 else 0, sc if C > 1 else d,
        _at(acc, "acc", torch.float32, B * G * C, dev), _at(pos, "pos", i32, B * G * C, dev),
        _at(length, "len", i32, B * G, dev), _at(seen, "seen", i32, B, dev))


def cache_append(cache, Q, K, V, *, L, rows=None, freq=None, interleaved=False, mscale=1.0, gamma_q=None, gamma_k=None,
                 eps=1e-6, out=None, workspace=None, stream=None):
    """``sc_cache_append``: Q [B*L, H * d] (None: no queries), K and V [B*L, Hk * d] (row strides multiples of 8) of
    up to L tokens a sequence.  Returns dict(Q, len, seen): the rotated queries, and len and seen moved on,
    which are the cache's own unless ``out`` has others.  ``workspace_status`` of the workspace reports a cache that was
    full: without a workspace of the caller's nothing does."""
    dev = _device(K, "K")
    (B, Hk, C, G, d, dt), view = _cache_at(cache, dev)
    T = B * L
    q, H, ldq = _heads_at(Q, "Q", dt, T, d, dev)
    k, hk, ldk = _heads_at(K, "K", dt, T, d, dev)
    v, hv, ldv = _heads_at(V, "V", dt, T, d, dev)
    if hk != Hk or hv != Hk:
        _refuse("K, V: the cache's heads are wanted")
    if out is None or (H and "Q" not in out):
        out = _rest(out, [("Q", (T, H * d), dt)] if H else [], K.device, stream)
    if "len" not in out or "seen" not in out:
        out = {"len": cache["len"], "seen": cache["seen"], **out}
    qo, ho, ldqo = _heads_at(out["Q"] if H else None, "out Q", dt, T, d, dev)
    _same(ho, H, "out Q")
    gq, gk, rot, f = _turn_at(freq, gamma_q, gamma_k, d, dev)
    i32 = torch.int32
    a = _APPEND.pack(B, C, H, Hk, G, *view, L, q, ldq, k, ldk, v, ldv, _at(rows, "rows", i32, B, dev), gq, gk, eps, rot,
                     1 if interleaved else 0, f, mscale, qo, ldqo, _at(out["len"], "out len", i32, B * G, dev),
                     _at(out["seen"], "out seen", i32, B, dev))
    ws = workspace if workspace is not None else _own_work(_aligned(256, K.device), K.device, stream)
    _call(_APPEND, a, ws, dev, stream)
    return out


def cache_attend(cache, Q, *, T, rows=None, scale=None, decay=1.0, out=None, workspace=None, stream=None):
    """``sc_cache_attend``: Q [B*T, H * d] (a row stride that is a multiple of 8), the rotated queries of the tokens that
    ``cache_append`` just brought; scale: 1 / sqrt(d) where None.  Returns dict(O [B*T, H * d], acc), acc being the
    cache's own unless ``out`` has another."""
    dev = _device(Q, "Q")
    (B, Hk, C, G, d, dt), view = _cache_at(cache, dev)
    q, H, ldq = _heads_at(Q, "Q", dt, B * T, d, dev)
    if out is None or "O" not in out:
        out = _rest(out, [("O", (B * T, H * d), dt)], Q.device, stream)
    if "acc" not in out:
        out = {"acc": cache["acc"], **out}
    o, ho, ldo = _heads_at(out["O"], "O", dt, B * T, d, dev)
    _same(ho, H, "O")
    a = _ATTEND.pack(B, C, H, Hk, G, *view, T, q, ldq, _at(rows, "rows", torch.int32, B, dev),
                     1 / math.sqrt(d) if scale is None else scale, decay, o, ldo,
                     _at(out["acc"], "out acc", torch.float32, B * G * C, dev))
    if workspace is None:
        workspace = _own_work(new_cache_workspace(B, C, H, Hk, width=d, lists=G, T=T, device=Q.device), Q.device, stream)
    _call(_ATTEND, a, workspace, dev, stream)
    return out


def cache_evict(cache, *, budget, slack=0, sinks=0, recent=0, out=None, workspace=None, stream=None):
    """``sc_cache_evict``: lists with more than budget + slack slots in use are brought down to budget.
    Returns dict(acc, pos, len), the cache's own unless ``out`` has others (K and V change in place)."""
    K = cache["K"]
    dev = _device(K, "K")
    (B, Hk, C, G, d, dt), view = _cache_at(cache, dev)
    if out is None or "acc" not in out or "pos" not in out or "len" not in out:
        out = {"acc": cache["acc"], "pos": cache["pos"], "len": cache["len"], **(out or {})}
    i32 = torch.int32
    a = _EVICT.pack(B, C, Hk, G, *view, budget, slack, sinks, recent, _at(out["acc"], "out acc", torch.float32, B * G * C, dev),
                    _at(out["pos"], "out pos", i32, B * G * C, dev), _at(out["len"], "out len", i32, B * G, dev))
    if workspace is None:
        workspace = _own_work(new_cache_workspace(B, C, Hk, Hk, width=d, lists=G, device=K.device), K.device, stream)
    _call(_EVICT, a, workspace, dev, stream)
    return out
