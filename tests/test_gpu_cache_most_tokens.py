"""One sequence of the most tokens that a call takes, into a cache with room for five: slot numbers of the last tokens would pass
2^31."""
import pytest
import torch

import paper_2310_07109_gb300 as sc

pytestmark = pytest.mark.gpu


def test_append_of_the_most_tokens():
    L, C, d = 2 ** 31 - 4096, sc.MAX_CACHE, 16
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GB")
    x = torch.empty(L, d, dtype=torch.bfloat16, device="cuda")   # keys and values both; of all but the first, anything
    x[:8] = torch.arange(8 * d, device="cuda").view(8, d)
    cache = sc.new_cache(1, C, 1, width=d)
    cache["len"].fill_(C - 5)
    cache["acc"].fill_(3.0)
    ws = sc.new_cache_workspace(1, C, 1, 1, width=d)
    sc.cache_append(cache, None, x, x, L=L, workspace=ws)
    assert sc.workspace_status(ws) == sc.SC_ERR_CAPACITY
    assert int(cache["len"]) == C and int(cache["seen"]) == L
    for n in ("K", "V"):
        assert torch.equal(cache[n][0, 0, C - 5:], x[:5]) and not bool(cache[n][0, 0, :C - 5].any()), n
    assert cache["pos"][0, 0, C - 5:].tolist() == [0, 1, 2, 3, 4] and not bool(cache["pos"][0, 0, :C - 5].any())
    assert not bool(cache["acc"][0, 0, C - 5:].any()) and bool((cache["acc"][0, 0, :C - 5] == 3).all())
    del x
    torch.cuda.empty_cache()
