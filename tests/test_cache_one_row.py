"""A single row has no distance to the next one: a view of one row of a matrix of any width will do.  Host tensors that name a
device; no GPU is reached."""
import pytest
import torch

import paper_2310_07109_gb300 as sc
from paper_2310_07109_gb300 import cache as ca
from test_cache_devices import On, d, no_library, on  # noqa: F401


def row(heads, width):
    """The first row of a matrix whose rows are `width` apart."""
    return torch.zeros(3, width, dtype=torch.bfloat16)[:1, :heads * d].as_subclass(On)


@pytest.mark.parametrize("width", [4 * d, 4 * d + 8, 4 * d + 3])
def test_a_row_of_a_wider_matrix(monkeypatch, width):
    seen = {}
    for name in ("_ROTATE", "_ROTATE_BACK", "_APPEND", "_ATTEND"):
        entry = getattr(ca, name)
        monkeypatch.setattr(entry, "call", lambda a, *_, e=entry: seen.update({e.name: e.args.from_buffer_copy(a)}) or 0)
    Q, K, ws = row(4, width), row(2, width), on(1 << 20, dtype=torch.uint8)
    cache = dict(K=on(1, 2, 32, d), V=on(1, 2, 32, d), acc=on(1, 1, 32, dtype=torch.float32), pos=on(1, 1, 32, dtype=torch.int32),
                 len=on(1, 1, dtype=torch.int32), seen=on(1, dtype=torch.int32))
    sc.rotate_forward(Q, K, width=d, B=1, L=1, out=dict(Q=row(4, width), K=row(2, width)))
    sc.rotate_backward(Q, K, width=d, B=1, L=1, out=dict(dQ=row(4, width), dK=row(2, width)), workspace=ws)
    sc.cache_append(cache, Q, K, K, L=1, out=dict(Q=row(4, width)), workspace=ws)
    sc.cache_attend(cache, Q, T=1, out=dict(O=row(4, width)), workspace=ws)
    assert len(seen) == 4
    for name, a in seen.items():
        for field in ("ldq", "ldq_out", "ldq_grad", "ldo"):
            # (backward's ldq is of Q, which there is none of)
            if hasattr(a, field) and not (name == "sc_rotate_backward" and field == "ldq"):
                assert getattr(a, field) == 4 * d, (name, field)
        for field in ("ldk", "ldk_out", "ldk_grad", "ldv"):
            if hasattr(a, field) and not (name == "sc_rotate_backward" and field == "ldk"):
                assert getattr(a, field) == 2 * d, (name, field)
