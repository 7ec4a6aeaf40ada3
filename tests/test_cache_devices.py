"""The rotation and cache calls run on the current device: tensors, a workspace or a stream of another
one are refused on the host, before the library is called, and so are wrong types and shapes.  The
devices are made up (host tensors that name one), so no GPU is needed and none is reached."""
import types

import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import cache as ca
from paper_2310_07109_gb300 import expert as ex

B, L, H, Hk, G, C, d = 2, 3, 4, 2, 2, 32, 64
T = B * L
i32, f32, bf = torch.int32, torch.float32, torch.bfloat16


class On(torch.Tensor):
    """A host tensor that says it lies on a cuda device (0 where none is set)."""
    at = 0
    is_cuda = True

    def get_device(self):
        return self.at


def on(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype).as_subclass(On)


def tensors():
    return types.SimpleNamespace(
        Q=on(T, H * d), K=on(T, Hk * d), V=on(T, Hk * d), dQ=on(T, H * d), dK=on(T, Hk * d), Qo=on(T, H * d), Ko=on(T, Hk * d),
        rows=on(B, dtype=i32), pos=on(B, L, dtype=i32), freq=on(d // 2, dtype=torch.float64), gq=on(d, dtype=f32), gk=on(d, dtype=f32),
        dgq=on(d, dtype=f32), dgk=on(d, dtype=f32), cK=on(B, Hk, C, d), cV=on(B, Hk, C, d), acc=on(B, G, C, dtype=f32),
        cpos=on(B, G, C, dtype=i32), len=on(B, G, dtype=i32), seen=on(B, dtype=i32), acc2=on(B, G, C, dtype=f32),
        pos2=on(B, G, C, dtype=i32), len2=on(B, G, dtype=i32), seen2=on(B, dtype=i32), ws=on(1 << 20, dtype=torch.uint8))


def cache(t):
    return dict(K=t.cK, V=t.cV, acc=t.acc, pos=t.cpos, len=t.len, seen=t.seen)


TURN = lambda t: dict(freq=t.freq, gamma_q=t.gq, gamma_k=t.gk)  # noqa: E731
IN_CACHE = ["cK", "cV", "acc", "cpos", "len", "seen"]
CALLS = {
    "rotate": (lambda t, **s: sc.rotate_forward(t.Q, t.K, width=d, B=B, L=L, rows=t.rows, pos=t.pos, out=dict(Q=t.Qo, K=t.Ko),
                                                **TURN(t), **s), ["Q", "K", "rows", "pos", "freq", "gq", "gk", "Qo", "Ko"]),
    "back": (lambda t, **s: sc.rotate_backward(t.dQ, t.dK, t.Q, t.K, width=d, B=B, L=L, rows=t.rows, pos=t.pos, workspace=t.ws,
                                               out=dict(dQ=t.Qo, dK=t.Ko, dgamma_q=t.dgq, dgamma_k=t.dgk), **TURN(t), **s),
             ["dQ", "dK", "Q", "K", "rows", "pos", "freq", "gq", "gk", "Qo", "Ko", "dgq", "dgk", "ws"]),
    "append": (lambda t, **s: sc.cache_append(cache(t), t.Q, t.K, t.V, L=L, rows=t.rows, workspace=t.ws,
                                              out=dict(Q=t.Qo, len=t.len2, seen=t.seen2), **TURN(t), **s),
               IN_CACHE + ["Q", "K", "V", "rows", "freq", "gq", "gk", "Qo", "len2", "seen2", "ws"]),
    "attend": (lambda t, **s: sc.cache_attend(cache(t), t.Q, T=L, rows=t.rows, workspace=t.ws, out=dict(O=t.Qo, acc=t.acc2), **s),
               IN_CACHE + ["Q", "rows", "Qo", "acc2", "ws"]),
    "evict": (lambda t, **s: sc.cache_evict(cache(t), budget=8, workspace=t.ws, out=dict(acc=t.acc2, pos=t.pos2, len=t.len2), **s),
              IN_CACHE + ["acc2", "pos2", "len2", "ws"]),
}


class Reached(Exception):
    """The library would have been called."""


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def reached(*_):
        raise Reached

    for name in ("_ROTATE", "_ROTATE_BACK", "_APPEND", "_ATTEND", "_EVICT"):
        monkeypatch.setattr(getattr(ca, name), "call", reached)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0)
    monkeypatch.setattr(ex, "_current_device", lambda: 0, raising=False)


def refused(call):
    with pytest.raises(sc.SparseCoderError) as e:
        call()
    assert e.value.code == sc.SC_ERR_INVALID_ARG


@pytest.mark.parametrize("what", list(CALLS))
def test_one_device(what):
    with pytest.raises(Reached):
        CALLS[what][0](tensors())


@pytest.mark.parametrize("what", list(CALLS))
def test_all_on_another_device(what):
    t = tensors()
    for v in vars(t).values():
        v.at = 1
    refused(lambda: CALLS[what][0](t))


@pytest.mark.parametrize("what,name", [(w, n) for w, (_, names) in CALLS.items() for n in names])
@pytest.mark.parametrize("device", [1, -1])   # -1: a host tensor
def test_one_tensor_elsewhere(what, name, device):
    t = tensors()
    getattr(t, name).at = device
    refused(lambda: CALLS[what][0](t))


@pytest.mark.parametrize("what,name", [(w, n) for w, (_, names) in CALLS.items() for n in names if n != "ws"])
def test_one_tensor_of_another_type_or_shape(what, name):
    t = tensors()
    old = getattr(t, name)
    setattr(t, name, on(*old.shape, dtype=torch.int64))
    refused(lambda: CALLS[what][0](t))
    wide = list(old.shape)
    wide[0] += 1
    if name in ("Q", "K", "V", "dQ", "dK", "Qo", "Ko", "cK", "cV") or old.dim() == 1 or name.startswith(("acc", "pos", "cpos", "len")):
        if name != "freq":   # (any number of frequencies up to half of the width)
            setattr(t, name, on(*wide, dtype=old.dtype))
            refused(lambda: CALLS[what][0](t))


def test_heads_and_strides():
    t = tensors()
    for name, bad in (("Q", on(T, H * d - 8)), ("K", on(T, d)), ("V", on(T, 3 * d)), ("Qo", on(T, d)), ("Q", on(T * H * d)),
                      ("cV", on(B, Hk, C + 1, d)[:, :, 1:]), ("cK", on(B, Hk, d, C).transpose(2, 3)), ("cK", on(B, Hk, C, d, dtype=torch.float16)),
                      ("K", on(T, Hk * d, dtype=torch.float16))):
        t = tensors()
        setattr(t, name, bad)
        refused(lambda: CALLS["append"][0](t))


@pytest.mark.parametrize("what", list(CALLS))
def test_a_stream_of_another_device(what):
    stream = types.SimpleNamespace(device_index=1, cuda_stream=0)
    refused(lambda: CALLS[what][0](tensors(), stream=stream))
    stream.device_index = 0
    with pytest.raises(Reached):
        CALLS[what][0](tensors(), stream=stream)


def test_outputs_that_are_not_named_are_made(monkeypatch):
    """Any part of ``out`` may be left out; of what is there, nothing is replaced."""
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: on(*([shape] if isinstance(shape, int) else shape), dtype=dtype))
    for what in CALLS:
        monkeypatch.setattr(getattr(ca, {"rotate": "_ROTATE", "back": "_ROTATE_BACK", "append": "_APPEND", "attend": "_ATTEND",
                                         "evict": "_EVICT"}[what]), "call", lambda *_: 0)
    t = tensors()
    c = cache(t)
    whole = {
        "rotate": (lambda out: sc.rotate_forward(t.Q, t.K, width=d, B=B, L=L, out=out, **TURN(t)), dict(Q=t.Qo, K=t.Ko)),
        "back": (lambda out: sc.rotate_backward(t.dQ, t.dK, t.Q, t.K, width=d, B=B, L=L, workspace=t.ws, out=out, **TURN(t)),
                 dict(dQ=t.Qo, dK=t.Ko, dgamma_q=t.dgq, dgamma_k=t.dgk)),
        "append": (lambda out: sc.cache_append(c, t.Q, t.K, t.V, L=L, workspace=t.ws, out=out), dict(Q=t.Qo, len=t.len2, seen=t.seen2)),
        "attend": (lambda out: sc.cache_attend(c, t.Q, T=L, workspace=t.ws, out=out), dict(O=t.Qo, acc=t.acc2)),
        "evict": (lambda out: sc.cache_evict(c, budget=8, workspace=t.ws, out=out), dict(acc=t.acc2, pos=t.pos2, len=t.len2)),
    }
    for what, (call, names) in whole.items():
        for n in range(2 ** len(names)):
            given = {name: v for i, (name, v) in enumerate(names.items()) if n >> i & 1}
            before = dict(given)
            got = call(given)
            assert list(given) == list(before)
            assert set(got) == set(names)
            for name, v in names.items():
                if name in given:
                    assert got[name] is v, (what, name)
                elif name in ("len", "seen", "acc", "pos"):
                    assert got[name] is c[name], (what, name)
                else:
                    assert got[name] is not v and got[name].shape == v.shape and got[name].dtype == v.dtype, (what, name)
        assert set(call(None)) == set(names)
