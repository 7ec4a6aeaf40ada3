"""Refusals of the expert feed-forward calls: arguments are checked on the host before
anything is launched, so these calls never reach a device."""
import ctypes
import os
import re

import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import build as bld
from paper_2310_07109_gb300 import expert as ex

FAKE = 1 << 40   # never dereferenced by the checks
P = FAKE
BIG = 1 << 30
OK = dict(
    route=(ex.RouteArgs, "sc_expert_route_forward", True,
           dict(B=2, L=64, E=16, k=2, logits=P, ld=16, rows=None, renormalize=1, expert=P, gate=P, offsets=P,
                slot=P, token=P)),
    route_back=(ex.RouteBackwardArgs, "sc_expert_route_backward", False,
                dict(B=2, L=64, E=16, k=2, logits=P, ld=16, rows=None, renormalize=1, expert=P, gate=P, dgate=P,
                     dlogits=P)),
    linear=(ex.ExpertLinearArgs, "sc_expert_linear_forward", True,
            dict(M=100, E=4, N=64, K=128, X=P, ldx=128, x_rows=100, token=None, offsets=P, W=P, bias=None, gelu=0,
                 pre=None, out=P, out_f32=0)),
    back_x=(ex.ExpertLinearBackwardInputArgs, "sc_expert_linear_backward_input", True,
            dict(M=100, E=4, N=64, K=128, dY=P, ldy=64, offsets=P, W=P, pre=None, dX=P, out_f32=0)),
    back_w=(ex.ExpertLinearBackwardWeightArgs, "sc_expert_linear_backward_weight", True,
            dict(M=100, E=4, N=64, K=128, dY=P, ldy=64, X=P, ldx=128, x_rows=100, token=None, offsets=P, dW=P,
                 out_f32=1, dbias=None)),
    combine=(ex.ExpertCombineArgs, "sc_expert_combine_forward", False,
             dict(B=2, L=64, D=128, k=2, M=256, rows=None, Y=P, slot=P, gate=P, res=P, res_scale=1.0, gamma=P,
                  beta=P, eps=1e-5, sum=P, out=P)),
    combine_back=(ex.ExpertCombineBackwardArgs, "sc_expert_combine_backward", True,
                  dict(B=2, L=64, D=128, k=2, M=256, rows=None, Y=P, slot=P, gate=P, res=P, res_scale=1.0, gamma=P,
                       eps=1e-5, dout=P, dsum=None, dY=P, dgate=P, dres=P, dgamma=P, dbeta=P)),
)
INVALID, UNSUPPORTED, WORKSPACE = sc.SC_ERR_INVALID_ARG, sc.SC_ERR_UNSUPPORTED, sc.SC_ERR_WORKSPACE
BAD = {
    "route": [(dict(B=0), INVALID), (dict(L=-1), INVALID), (dict(E=0), INVALID), (dict(k=0), INVALID),
              (dict(k=17), INVALID), (dict(k=9), UNSUPPORTED), (dict(E=257, ld=300), UNSUPPORTED), (dict(ld=15), INVALID),
              (dict(B=1 << 20, L=1 << 11), INVALID), (dict(logits=None), INVALID), (dict(expert=None), INVALID),
              (dict(gate=None), INVALID), (dict(offsets=None), INVALID), (dict(slot=None), INVALID),
              (dict(token=None), INVALID)],
    "route_back": [(dict(B=0), INVALID), (dict(k=17), INVALID), (dict(E=257, ld=300), UNSUPPORTED), (dict(ld=3), INVALID),
                   (dict(logits=None), INVALID), (dict(expert=None), INVALID), (dict(gate=None), INVALID),
                   (dict(dgate=None), INVALID), (dict(dlogits=None), INVALID)],
    "linear": [(dict(M=0), INVALID), (dict(E=0), INVALID), (dict(E=257), UNSUPPORTED), (dict(N=60), INVALID),
               (dict(K=4, ldx=8), INVALID), (dict(N=8200), UNSUPPORTED), (dict(ldx=120), INVALID), (dict(ldx=132), INVALID),
               (dict(x_rows=99), INVALID), (dict(token=P, x_rows=0), INVALID), (dict(X=None), INVALID),
               (dict(X=P + 8), INVALID), (dict(W=None), INVALID), (dict(W=P + 2), INVALID), (dict(offsets=None), INVALID),
               (dict(out=None), INVALID), (dict(out=P + 4), INVALID), (dict(pre=P + 2), INVALID)],
    "back_x": [(dict(M=0), INVALID), (dict(N=12), INVALID), (dict(K=8200), UNSUPPORTED), (dict(ldy=56), INVALID),
               (dict(dY=None), INVALID), (dict(dY=P + 2), INVALID), (dict(W=None), INVALID), (dict(offsets=None), INVALID),
               (dict(dX=None), INVALID), (dict(dX=P + 8), INVALID), (dict(pre=P + 8), INVALID)],
    "back_w": [(dict(E=-3), INVALID), (dict(ldy=56), INVALID), (dict(ldx=12), INVALID), (dict(x_rows=99), INVALID),
               (dict(token=P, x_rows=0), INVALID), (dict(dY=None), INVALID), (dict(X=None), INVALID),
               (dict(offsets=None), INVALID), (dict(dW=None), INVALID), (dict(dW=P + 8), INVALID)],
    "combine": [(dict(B=0), INVALID), (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(D=12), INVALID),
                (dict(D=8200), UNSUPPORTED), (dict(M=0), INVALID), (dict(Y=None), INVALID), (dict(Y=P + 8), INVALID),
                (dict(slot=None), INVALID), (dict(res=P + 2), INVALID), (dict(beta=None), INVALID),
                (dict(gamma=None), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
                (dict(out=None), INVALID), (dict(gamma=None, beta=None, sum=None), INVALID), (dict(sum=P + 8), INVALID)],
    "combine_back": [(dict(L=0), INVALID), (dict(D=8200), UNSUPPORTED), (dict(dY=None), INVALID), (dict(dout=None), INVALID),
                     (dict(dgamma=None), INVALID), (dict(dbeta=None), INVALID), (dict(gamma=None), INVALID),
                     (dict(gamma=None, dout=None, dgamma=None, dbeta=None), INVALID), (dict(dY=P + 8), INVALID),
                     (dict(dsum=P + 2), INVALID), (dict(dres=P + 2), INVALID), (dict(eps=-1.0), INVALID)],
}


@pytest.fixture(scope="module")
def lib():
    bld.build_library()
    return ex._library()


def call(lib, what, ws=FAKE, ws_bytes=BIG, **kw):
    struct, name, with_ws, args = OK[what]
    a = struct(**{**args, **kw})
    return getattr(lib, name)(a, ws, ws_bytes, None) if with_ws else getattr(lib, name)(a, None)


@pytest.mark.parametrize("what,kw,code", [(w, kw, c) for w, cases in BAD.items() for kw, c in cases])
def test_bad_arguments(lib, what, kw, code):
    assert call(lib, what, **kw) == code


WORDS = {   # arrays of 32-bit values
    "route": ("logits", "rows", "expert", "gate", "offsets", "slot", "token"),
    "route_back": ("logits", "rows", "expert", "gate", "dgate", "dlogits"),
    "linear": ("token", "offsets", "bias"), "back_x": ("offsets",), "back_w": ("token", "offsets", "dbias"),
    "combine": ("rows", "slot", "gate", "gamma", "beta"),
    "combine_back": ("rows", "slot", "gate", "gamma", "dgate", "dgamma", "dbeta"),
}


@pytest.mark.parametrize("what,name", [(w, n) for w, names in WORDS.items() for n in names])
def test_words_lie_at_multiples_of_four(lib, what, name):
    for by in (1, 2, 3):
        assert call(lib, what, **{name: P + by}) == INVALID


def test_most_slots(lib):
    most = 2 ** 31 - 4096
    for what in ("linear", "back_x", "back_w"):
        rows = {} if what == "back_x" else dict(x_rows=2 ** 31 - 1)
        assert call(lib, what, M=most + 1, **rows) == UNSUPPORTED
        assert call(lib, what, M=most, ws=None, **rows) == WORKSPACE   # (the last check)
    assert call(lib, "route", B=1, L=most // 2 + 1) == INVALID
    assert call(lib, "route", B=1, L=most // 2, ws=None) == WORKSPACE
    assert sc.expert_workspace_size(1, most + 1, 4, 1, 8) == 0 < sc.expert_workspace_size(1, most, 4, 1, 8)


@pytest.mark.parametrize("what", list(OK))
def test_missing_arguments(lib, what):
    _, name, with_ws, _ = OK[what]
    assert (getattr(lib, name)(None, FAKE, BIG, None) if with_ws else getattr(lib, name)(None, None)) == INVALID


@pytest.mark.parametrize("what", [w for w, v in OK.items() if v[2]])
def test_bad_workspace(lib, what):
    for ws, size in ((None, BIG), (FAKE + 128, BIG), (FAKE, 16)):
        assert call(lib, what, ws=ws, ws_bytes=size) == WORKSPACE


def test_workspace_size(lib):
    assert sc.expert_workspace_size(8, 1024, 16, 2, 768) % 256 == 0
    assert sc.expert_workspace_size(8, 1024, 16, 2, 1024) > sc.expert_workspace_size(8, 1024, 16, 2, 768) > 0
    for bad in ((0, 1, 1, 1, 8), (1, 0, 1, 1, 8), (1, 1, 0, 1, 8), (1, 1, 257, 1, 8), (1, 1, 4, 5, 8), (1, 1, 16, 9, 8),
                (1, 1, 4, 2, 12), (1, 1, 4, 2, 8200), (1 << 20, 1 << 11, 4, 2, 8)):
        assert sc.expert_workspace_size(*bad) == 0


def test_constants_and_structs_match_the_header():
    text = open(os.path.join(bld.INCLUDE, "sparsecoder.h")).read()
    d = dict(re.findall(r"^#define\s+(SC_\w+)\s+(\d+)", text, re.M))
    assert (int(d["SC_MAX_EXPERTS"]), int(d["SC_MAX_CHOICES"]), int(d["SC_MAX_EXPERT_DIM"])) == (
        sc.MAX_EXPERTS, sc.MAX_CHOICES, sc.MAX_EXPERT_DIM)
    for struct, name, _, _ in OK.values():
        body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name.replace("_forward", "").replace(
            "sc_expert_linear", "sc_expert_linear").__add__("_args"), text)
        assert body, name
        fields = [f.strip(" *") for line in body.group(1).split(";") if line.strip()
                  for f in re.sub(r"^\s*(const )?(long long|\w+)\s*\*?", "", line.strip()).split(",")]
        assert fields == [f[0] for f in struct._fields_], name


def test_the_binding_refuses_wrong_tensors():
    """Types, shapes and host tensors, before the library is called."""
    cpu = torch.zeros(4, 8)
    for call in (lambda: sc.expert_route_forward(cpu, k=2, B=1, L=4),
                 lambda: sc.expert_linear_forward(cpu.bfloat16(), torch.zeros(1, 8, 8).bfloat16(), cpu),
                 lambda: sc.expert_combine_forward(cpu.bfloat16(), cpu.int(), B=1, L=4)):
        with pytest.raises(sc.SparseCoderError) as e:
            call()
        assert e.value.code == INVALID


def test_the_binding_refuses_wrong_dimensions():
    bf = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)  # noqa: E731
    one = torch.zeros((), dtype=torch.int32)
    for call in (lambda: ex._shape(bf(8, 8), "W", 3), lambda: ex._shape(one, "offsets", 1),
                 lambda: sc.expert_combine_forward(bf(4, 8, 1), one, B=1, L=4),
                 lambda: sc.expert_combine_backward(bf(4, 8), torch.zeros(4, dtype=torch.int32), B=1, L=4)):
        with pytest.raises(sc.SparseCoderError) as e:
            call()
        assert e.value.code == INVALID
