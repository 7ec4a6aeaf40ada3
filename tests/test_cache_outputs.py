"""What the binding makes of ``out``: names that a call does not know are left alone.  Host tensors that name a device; no GPU
is reached."""
import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import cache as ca
from test_cache_devices import cache, no_library, tensors  # noqa: F401


@pytest.mark.parametrize("names", [("Q", "O", "acc"), ("Q", "O", "seen"), ("Q", "O", "acc", "pos"), ("Q", "O", "seen", "len"), ("Q", "O", "seen", "more", "acc")])
def test_one_dict_for_all_calls_of_a_step(monkeypatch, names):
    """Eviction completes it by its names, whatever else it holds."""
    monkeypatch.setattr(ca._EVICT, "call", lambda *_: 0)
    t = tensors()
    c = cache(t)
    mine = {"acc": t.acc2, "pos": t.pos2, "len": t.len2}
    out = {n: mine.get(n, torch.zeros(1)) for n in names}
    got = sc.cache_evict(c, budget=8, workspace=t.ws, out=out)
    for n in ("acc", "pos", "len"):
        assert got[n] is (out[n] if n in out else c[n]), n
    assert all(got[n] is out[n] for n in names)
