"""Outputs in the place of the inputs keep the inputs' distances: other ones, by which tokens would be written over before they
are read, are refused on the host.  One token has no distance."""
import pytest

import paper_2310_07109_gb300 as sc
from test_abi_cache import P, call, lib  # noqa: F401

FAR = P + (1 << 20)
APART = {"rotate": dict(Q=P, K=FAR, Q_out=P, K_out=FAR), "back": dict(dQ_out=P, dK_out=FAR, dQ=P, dK=FAR), "append": dict(Q=P, Q_out=P)}


@pytest.mark.parametrize("what,kw", [("rotate", dict(ldq_out=264)), ("rotate", dict(ldk_out=256)), ("rotate", dict(ldq=512)), ("rotate", dict(ldk=136)),
                                     ("back", dict(ldq_grad=264)), ("back", dict(ldk_grad=256)), ("back", dict(ldq_out=264)), ("back", dict(ldk_out=136)),
                                     ("append", dict(ldq_out=520)), ("append", dict(ldq=1024))])
def test_other_distances_are_refused(lib, what, kw):  # noqa: F811
    assert call(lib, what, **{**APART[what], **kw}) == sc.SC_ERR_INVALID_ARG


@pytest.mark.parametrize("what", ["back", "append"])
def test_the_inputs_own_distances_are_not(lib, what):  # noqa: F811
    """(the workspace is looked at last: what comes before it has passed)"""
    ld = {"back": dict(ldq_out=512, ldq_grad=512, ldk_out=256, ldk_grad=256), "append": dict(ldq=1024, ldq_out=1024)}[what]
    assert call(lib, what, ws=None, **{**APART[what], **ld}) == sc.SC_ERR_WORKSPACE


@pytest.mark.parametrize("what", ["back", "append"])
def test_one_token_has_no_distance(lib, what):  # noqa: F811
    ld = {"back": dict(ldq_grad=512, ldk_grad=1024), "append": dict(ldq_out=1024)}[what]
    assert call(lib, what, ws=None, **{**APART[what], **ld, "B": 1, "L": 1}) == sc.SC_ERR_WORKSPACE
