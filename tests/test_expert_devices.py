"""The expert feed-forward calls run on the current device: tensors, a workspace or a stream
of another one are refused on the host, before the library is called.  The devices are
made up (host tensors that name one), so no GPU is needed and none is reached."""
import types

import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import expert as ex

B, L, E, K_CHOICES, D, F = 1, 4, 4, 2, 16, 24
T, M = B * L, B * L * K_CHOICES


class On(torch.Tensor):
    """A host tensor that says it lies on a cuda device (0 where none is set)."""
    at = 0
    is_cuda = True

    def get_device(self):
        return self.at


def on(device, *shape, dtype=torch.bfloat16):
    t = torch.zeros(shape, dtype=dtype).as_subclass(On)
    t.at = device
    return t


def tensors():
    i32, f32 = torch.int32, torch.float32
    t = dict(logits=on(0, T, E, dtype=f32), rows=on(0, B, dtype=i32), expert=on(0, T, K_CHOICES, dtype=i32),
             gate=on(0, T, K_CHOICES, dtype=f32), dgate=on(0, T, K_CHOICES, dtype=f32), offsets=on(0, E + 1, dtype=i32),
             slot=on(0, T, K_CHOICES, dtype=i32), token=on(0, M, dtype=i32), dlogits=on(0, T, E, dtype=f32),
             X=on(0, T, D), W=on(0, E, F, D), bias=on(0, E, F, dtype=f32), pre=on(0, M, F), out=on(0, M, F),
             dY=on(0, M, F), pre_in=on(0, M, D), dX=on(0, M, D), dW=on(0, E, F, D, dtype=f32),
             dbias=on(0, E, F, dtype=f32), Y=on(0, M, D), res=on(0, T, D), gamma=on(0, D, dtype=f32),
             beta=on(0, D, dtype=f32), sum=on(0, T, D), norm=on(0, T, D), dout=on(0, T, D), dsum=on(0, T, D),
             dYs=on(0, M, D), dres=on(0, T, D), dgamma=on(0, D, dtype=f32), dbeta=on(0, D, dtype=f32),
             ws=on(0, 1 << 16, dtype=torch.uint8))
    return types.SimpleNamespace(**t)


CALLS = {
    "route": (lambda t, **s: sc.expert_route_forward(
        t.logits, k=K_CHOICES, B=B, L=L, rows=t.rows, workspace=t.ws,
        out=dict(expert=t.expert, gate=t.gate, offsets=t.offsets, slot=t.slot, token=t.token), **s),
        ["logits", "rows", "expert", "gate", "offsets", "slot", "token", "ws"]),
    "route_back": (lambda t, **s: sc.expert_route_backward(
        t.logits, t.expert, t.gate, t.dgate, B=B, L=L, rows=t.rows, out=t.dlogits, **s),
        ["logits", "expert", "gate", "dgate", "rows", "dlogits"]),
    "linear": (lambda t, **s: sc.expert_linear_forward(
        t.X, t.W, t.offsets, token=t.token, bias=t.bias, gelu=True, pre=t.pre, out=t.out, workspace=t.ws, **s),
        ["X", "W", "offsets", "token", "bias", "pre", "out", "ws"]),
    "back_x": (lambda t, **s: sc.expert_linear_backward_input(
        t.dY, t.W, t.offsets, pre=t.pre_in, out=t.dX, workspace=t.ws, **s),
        ["dY", "W", "offsets", "pre_in", "dX", "ws"]),
    "back_w": (lambda t, **s: sc.expert_linear_backward_weight(
        t.dY, t.X, t.offsets, token=t.token, out=dict(dW=t.dW, dbias=t.dbias), workspace=t.ws, **s),
        ["dY", "X", "offsets", "token", "dW", "dbias", "ws"]),
    "combine": (lambda t, **s: sc.expert_combine_forward(
        t.Y, t.slot, t.gate, B=B, L=L, rows=t.rows, res=t.res, gamma=t.gamma, beta=t.beta,
        out=dict(sum=t.sum, out=t.norm), **s),
        ["Y", "slot", "gate", "rows", "res", "gamma", "beta", "sum", "norm"]),
    "combine_back": (lambda t, **s: sc.expert_combine_backward(
        t.Y, t.slot, t.gate, B=B, L=L, rows=t.rows, res=t.res, gamma=t.gamma, dout=t.dout, dsum=t.dsum, workspace=t.ws,
        out=dict(dY=t.dYs, dgate=t.dgate, dres=t.dres, dgamma=t.dgamma, dbeta=t.dbeta), **s),
        ["Y", "slot", "gate", "rows", "res", "gamma", "dout", "dsum", "dYs", "dgate", "dres", "dgamma", "dbeta", "ws"]),
}


class Reached(Exception):
    """The library was called."""


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def reached(*_):
        raise Reached

    for name in ("_ROUTE", "_ROUTE_BACK", "_LINEAR", "_BACK_X", "_BACK_W", "_COMBINE", "_COMBINE_BACK"):
        monkeypatch.setattr(getattr(ex, name), "call", reached)
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


@pytest.mark.parametrize("what", list(CALLS))
def test_a_stream_of_another_device(what):
    stream = types.SimpleNamespace(device_index=1, cuda_stream=0)
    refused(lambda: CALLS[what][0](tensors(), stream=stream))
    stream.device_index = 0
    with pytest.raises(Reached):
        CALLS[what][0](tensors(), stream=stream)
