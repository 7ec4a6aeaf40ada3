"""Refusals of the rotation and cache calls: arguments are checked on the host before anything
is launched, so these calls never reach a device."""
import math
import os
import re

import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import build as bld
from paper_2310_07109_gb300 import cache as ca

P = 1 << 40   # never dereferenced by the checks
BIG = 1 << 40
INVALID, UNSUPPORTED, WORKSPACE = sc.SC_ERR_INVALID_ARG, sc.SC_ERR_UNSUPPORTED, sc.SC_ERR_WORKSPACE
TURN = dict(gamma_q=P, gamma_k=P, eps=1e-6, rot=64, interleaved=0, freq=P, mscale=1.0)
CACHE = dict(B=2, C=1000, Hk=4, G=2, d=64, dtype=0, K=P, V=P, stride_b=256000, stride_h=64000, stride_c=64, acc=P, pos=P,
             len=P, seen=P)
OK = dict(
    rotate=(ca.RotateArgs, "sc_rotate_forward", False,
            dict(B=2, L=10, Hq=4, Hk=2, d=64, dtype=1, Q=P, ldq=256, K=P, ldk=128, rows=None, pos=None, **TURN, Q_out=P,
                 ldq_out=256, K_out=P, ldk_out=128)),
    back=(ca.RotateBackwardArgs, "sc_rotate_backward", True,
          dict(B=2, L=10, Hq=4, Hk=2, d=64, dtype=0, dQ_out=P, ldq_out=256, dK_out=P, ldk_out=128, Q=P, ldq=256, K=P, ldk=128,
               rows=None, pos=None, **TURN, dQ=P, ldq_grad=256, dK=P, ldk_grad=128, dgamma_q=P, dgamma_k=P)),
    append=(ca.CacheAppendArgs, "sc_cache_append", True,
            dict(**CACHE, H=8, L=3, Q=P, ldq=512, K_in=P, ldk=256, V_in=P, ldv=256, rows=None, **TURN, Q_out=P, ldq_out=512,
                 len_out=P, seen_out=P)),
    attend=(ca.CacheAttendArgs, "sc_cache_attend", True,
            dict(**CACHE, H=8, T=3, Q=P, ldq=512, rows=None, scale=0.125, decay=1.0, O=P + 4096, ldo=512, acc_out=P)),
    evict=(ca.CacheEvictArgs, "sc_cache_evict", True,
           dict(**CACHE, budget=100, slack=0, sinks=4, recent=50, acc_out=P, pos_out=P, len_out=P)),
)
BAD_TURN = [(dict(B=0), INVALID), (dict(L=0), INVALID), (dict(d=0), INVALID), (dict(d=40), INVALID),
            (dict(rot=-16), INVALID), (dict(rot=24), INVALID), (dict(rot=80), INVALID), (dict(freq=None), INVALID),
            (dict(freq=P + 4), INVALID), (dict(mscale=math.inf), INVALID), (dict(mscale=math.nan), INVALID), (dict(eps=0.0), INVALID),
            (dict(eps=math.nan), INVALID), (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID)]
BAD_CACHE = [(dict(B=0), INVALID), (dict(C=0), INVALID), (dict(Hk=0), INVALID), (dict(G=3), INVALID), (dict(G=0), INVALID),
             (dict(C=262145), UNSUPPORTED), (dict(dtype=5), INVALID), (dict(K=None), INVALID), (dict(V=None), INVALID),
             (dict(K=P + 8), INVALID), (dict(V=P + 2), INVALID), (dict(stride_b=256004), INVALID), (dict(stride_h=4), INVALID),
             (dict(stride_h=0), INVALID), (dict(stride_b=-256000), INVALID), (dict(stride_c=56), INVALID), (dict(acc=None), INVALID),
             (dict(pos=None), INVALID), (dict(len=None), INVALID), (dict(seen=None), INVALID)]
BAD = {
    "rotate": BAD_TURN + [
        (dict(Hq=-1), INVALID), (dict(Hq=0, Hk=0), INVALID), (dict(Hq=1000, ldq=64000, ldq_out=64000, Hk=25, ldk=1600, ldk_out=1600), UNSUPPORTED),
        (dict(d=272, ldq=2048, ldk=2048), UNSUPPORTED), (dict(B=1 << 20, L=1 << 11), UNSUPPORTED), (dict(Q=None), INVALID),
        (dict(Q=P + 8), INVALID), (dict(ldq=248), INVALID), (dict(ldq=260), INVALID), (dict(ldq=1 << 30), INVALID),
        (dict(K=None), INVALID), (dict(Q_out=None), INVALID), (dict(K_out=P + 2), INVALID), (dict(ldk_out=120), INVALID)],
    "back": BAD_TURN + [
        (dict(Hk=-2), INVALID), (dict(dQ_out=None), INVALID), (dict(dK_out=P + 4), INVALID), (dict(Q=None), INVALID),
        (dict(K=None), INVALID), (dict(dQ=None), INVALID), (dict(dK=None), INVALID), (dict(ldq=100), INVALID), (dict(ldk_grad=64), INVALID),
        (dict(dgamma_q=None), INVALID), (dict(gamma_k=None), INVALID)],
    "append": BAD_TURN + BAD_CACHE + [
        (dict(H=6), INVALID), (dict(H=-4), INVALID), (dict(Q=None), INVALID), (dict(Q_out=None), INVALID), (dict(K_in=None), INVALID),
        (dict(V_in=P + 8), INVALID), (dict(ldv=248), INVALID), (dict(len_out=None), INVALID), (dict(seen_out=None), INVALID)],
    "attend": BAD_CACHE + [
        (dict(H=0), INVALID), (dict(H=6), INVALID), (dict(T=0), INVALID), (dict(T=4097), UNSUPPORTED), (dict(d=80, stride_c=80), UNSUPPORTED),
        (dict(d=32), UNSUPPORTED), (dict(Q=None), INVALID), (dict(ldq=504), INVALID), (dict(O=None), INVALID), (dict(O=P + 8), INVALID), (dict(O=P), INVALID),
        (dict(ldo=516), INVALID), (dict(acc_out=None), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID),
        (dict(decay=math.nan), INVALID)],
    "evict": BAD_CACHE + [
        (dict(budget=0), INVALID), (dict(slack=-1), INVALID), (dict(sinks=-1), INVALID), (dict(recent=-1), INVALID),
        (dict(recent=97), INVALID), (dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), INVALID), (dict(acc_out=None), INVALID),
        (dict(pos_out=None), INVALID), (dict(len_out=None), INVALID)],
}
WORDS = {"rotate": ("rows", "pos", "gamma_q", "gamma_k"), "back": ("rows", "pos", "gamma_q", "gamma_k", "dgamma_q", "dgamma_k"),
         "append": ("acc", "pos", "len", "seen", "rows", "gamma_q", "gamma_k", "len_out", "seen_out"),
         "attend": ("acc", "pos", "len", "seen", "rows", "acc_out"),
         "evict": ("acc", "pos", "len", "seen", "acc_out", "pos_out", "len_out")}


@pytest.fixture(scope="module")
def lib():
    bld.build_library()
    return ca._library()


def call(lib, what, ws=P, ws_bytes=BIG, **kw):
    struct, name, with_ws, args = OK[what]
    a = struct(**{**args, **kw})
    return getattr(lib, name)(a, ws, ws_bytes, None) if with_ws else getattr(lib, name)(a, None)


@pytest.mark.parametrize("what,kw,code", [(w, kw, c) for w, cases in BAD.items() for kw, c in cases])
def test_bad_arguments(lib, what, kw, code):
    assert call(lib, what, **kw) == code


@pytest.mark.parametrize("what,name", [(w, n) for w, names in WORDS.items() for n in names])
def test_words_lie_at_multiples_of_four(lib, what, name):
    for by in (1, 2, 3):
        assert call(lib, what, **{name: P + by}) == INVALID


@pytest.mark.parametrize("what", list(OK))
def test_missing_arguments(lib, what):
    _, name, with_ws, _ = OK[what]
    assert (getattr(lib, name)(None, P, BIG, None) if with_ws else getattr(lib, name)(None, None)) == INVALID


@pytest.mark.parametrize("what", [w for w, v in OK.items() if v[2]])
def test_bad_workspace(lib, what):
    """(the last check: what comes before it has passed)"""
    for ws, size in ((None, BIG), (P + 128, BIG), (P, 16)):
        assert call(lib, what, ws=ws, ws_bytes=size) == WORKSPACE


def test_workspace_sizes(lib):
    assert sc.rotate_workspace_size(256) > sc.rotate_workspace_size(64) > 0 == sc.rotate_workspace_size(64) % 256
    for bad in (0, 8, 40, 272):
        assert sc.rotate_workspace_size(bad) == 0
    size = sc.cache_workspace_size
    assert size(2, 1000, 8, 4, lists=2, T=3) % 256 == 0 < size(2, 1000, 8, 4, lists=2, T=3)
    assert size(2, 1000, 8, 4, T=64) > size(2, 1000, 8, 4, T=1)
    assert size(2, 1000, 0, 4, width=80) > 0
    for bad in (dict(B=0), dict(C=0), dict(C=262145), dict(H=6), dict(heads=0), dict(lists=3), dict(lists=0), dict(T=0), dict(T=4097),
                dict(width=24), dict(width=272), dict(width=80, T=2)):
        kw = {**dict(B=2, C=1000, H=8, heads=4, width=64, lists=2, T=1), **bad}
        assert size(**kw) == 0, bad
    # what the calls ask for is what the size says
    for what, T in (("attend", 3), ("evict", 1)):
        need = size(2, 1000, 8, 4, lists=2, T=T)
        assert call(lib, what, ws_bytes=need, ws=P + 64) == WORKSPACE and call(lib, "attend", ws_bytes=need - 256, T=T) == WORKSPACE


def test_constants_and_structs_match_the_header():
    text = open(os.path.join(bld.INCLUDE, "sparsecoder.h")).read()
    d = dict(re.findall(r"^#define\s+(SC_\w+)\s+(\d+)", text, re.M))
    assert [int(d[n]) for n in ("SC_MAX_HEAD_WIDTH", "SC_MAX_HEADS", "SC_MAX_CACHE", "SC_MAX_STEP")] == [
        sc.MAX_HEAD_WIDTH, sc.MAX_HEADS, sc.MAX_CACHE, sc.MAX_STEP]
    assert int(re.search(r"SC_ERR_CAPACITY = (\d+)", text).group(1)) == sc.SC_ERR_CAPACITY
    for struct, name, _, _ in OK.values():
        body = re.search(r"typedef struct \{([^{}]*)\} %s_args;" % name.replace("_forward", ""), text)
        assert body, name
        fields = [f.strip(" *") for line in body.group(1).split(";") if line.strip()
                  for f in re.sub(r"^\s*(const )?(long long|\w+)\s*\*?", "", line.strip()).split(",")]
        assert fields == [f[0] for f in struct._fields_], name


def test_status_string():
    assert sc.status_string(sc.SC_ERR_CAPACITY).startswith("SC_ERR_CAPACITY")


def bad_calls():
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    cache = sc.new_cache(1, 16, 2, device="cpu")
    return [lambda: sc.rotate_forward(bf(4, 64), width=64, B=1, L=4), lambda: sc.rotate_forward(None, None, width=64, B=1, L=4),
            lambda: sc.rotate_backward(None, None, width=64, B=1, L=4), lambda: sc.rotate_backward(bf(4, 64), width=64, B=1, L=4),
            lambda: sc.cache_append(cache, None, bf(1, 128), bf(1, 128), L=1), lambda: sc.cache_attend(cache, bf(1, 128), T=1),
            lambda: sc.cache_evict(cache, budget=4)]


@pytest.mark.parametrize("i", range(7))
def test_the_binding_refuses_host_tensors(i):
    with pytest.raises(sc.SparseCoderError) as e:
        bad_calls()[i]()
    assert e.value.code == INVALID


def test_new_cache():
    c = sc.new_cache(3, 50, 6, width=128, lists=2, dtype=torch.float16, device="cpu")
    assert c["K"].shape == c["V"].shape == (3, 6, 50, 128) and c["K"].dtype == torch.float16
    assert c["acc"].shape == c["pos"].shape == (3, 2, 50) and c["len"].shape == (3, 2) and c["seen"].shape == (3,)


def test_rotary_frequencies():
    f, m = sc.rotary_frequencies(64, device="cpu")
    assert f.dtype == torch.float64 and m == 1.0 and f[0] == 1.0
    assert torch.allclose(f, 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32), rtol=1e-14)
    g, m = sc.rotary_frequencies(64, method="linear", factor=4.0, device="cpu")
    assert torch.equal(g, f / 4) and m == 1.0
    g, _ = sc.rotary_frequencies(64, method="base", factor=4.0, device="cpu")
    assert g[0] == 1.0 and abs(float(g[-1] * 4 / f[-1]) - 1) < 1e-12 and bool((g[1:] < f[1:]).all())
    g, m = sc.rotary_frequencies(64, method="parts", factor=4.0, length=4096, low=1.0, high=32.0, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.allclose(g[turns <= 1], f[turns <= 1] / 4, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    assert bool(((g < f) & (g > f / 4))[mid].all()) and abs(m - (1 + 0.1 * math.log(4))) < 1e-15
    for bad in (dict(rot=63), dict(rot=0), dict(rot=64, method="other"), dict(rot=64, method="parts"), dict(rot=64, factor=0.5),
                dict(rot=2, method="base", factor=2.0), dict(rot=64, method="parts", length=100, low=3.0, high=2.0)):
        with pytest.raises(sc.SparseCoderError):
            sc.rotary_frequencies(**bad, device="cpu")
