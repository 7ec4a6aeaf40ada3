"""A workspace for steps of at most T tokens serves every shorter step: its size never falls as T grows, and no call
asks for more.  (The calls' own needs do fall: with more rows there are fewer parts, and scores are no longer kept.)"""
import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import build as bld


@pytest.fixture(scope="module", autouse=True)
def library():
    bld.build_library()


# B, C, H, Hk, lists, d: with as many query heads as key heads, grouped ones, and more of them than a tile of rows
SHAPES = [(32, 8192, 16, 4, 1, 128), (1, 2048, 12, 12, 1, 64), (4, 8192, 16, 4, 4, 128), (1, 2048, 16, 16, 16, 64), (1, 131072, 16, 2, 2, 128),
          (3, 8192, 64, 4, 1, 64), (1, 300, 5, 5, 5, 64), (2, 2048, 200, 2, 1, 128), (1, 262144, 1, 1, 1, 64)]


@pytest.mark.parametrize("B,C,H,Hk,G,d", SHAPES)
def test_the_size_never_falls(B, C, H, Hk, G, d):
    before = 0
    for T in list(range(1, 1400)) + [1500, 2048, 3000, 4000, 4096]:
        size = sc.cache_workspace_size(B, C, H, Hk, lists=G, width=d, T=T)
        assert size % 256 == 0 and size >= before > -1, T
        before = size


@pytest.mark.gpu
@pytest.mark.parametrize("B,C,H,Hk,G,d,most", [(8, 2048, 16, 4, 1, 128, 9), (1, 2048, 12, 12, 1, 64, 900), (2, 4096, 16, 4, 4, 128, 64),
                                               (1, 5000, 2, 1, 1, 64, 2000)])
def test_shorter_steps_take_the_workspace_of_the_longest(B, C, H, Hk, G, d, most):
    """The same bits as with a workspace of their own; the bytes behind are not touched."""
    g = torch.Generator(device="cuda")
    g.manual_seed(most)
    randn = lambda *s: torch.randn(s, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    cache = dict(K=randn(B, Hk, C, d), V=randn(B, Hk, C, d), acc=torch.zeros(B, G, C, device="cuda"),
                 pos=torch.arange(C, dtype=torch.int32, device="cuda").expand(B, G, C).contiguous(),
                 len=torch.full((B, G), C, dtype=torch.int32, device="cuda"), seen=torch.full((B,), C, dtype=torch.int32, device="cuda"))
    size = sc.cache_workspace_size(B, C, H, Hk, lists=G, width=d, T=most)
    raw = torch.full((size + 512,), 77, dtype=torch.uint8, device="cuda")
    at = -raw.data_ptr() % 256
    ws = raw[at:at + size]
    ws.zero_()
    r = H // Hk
    steps = {1, 2, 16 // r, 16 // r + 1, 32 // r, 32 // r + 1, 64 // r, 64 // r + 1, 257, 300, 769, most - 1, most}
    for T in sorted(t for t in steps if 1 <= t <= most):
        Q = randn(B * T, H * d)
        got, want = (sc.cache_attend(cache, Q, T=T, workspace=w, out=dict(acc=torch.zeros_like(cache["acc"]))) for w in (ws, None))
        assert torch.equal(got["O"], want["O"]) and torch.equal(got["acc"], want["acc"]), T
        assert bool((raw[:at] == 77).all()) and bool((raw[at + size:] == 77).all()), T
    assert sc.workspace_status(ws) == sc.SC_OK
