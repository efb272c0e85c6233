"""Refusals of the embedding calls: every one before a launch."""
import pytest

import paper_2210_00129_b200 as sbp
from paper_2210_00129_b200 import build as sbp_build

P = 0x1000          # never dereferenced
INV, UNS, WS = sbp.SBP_ERR_INVALID_ARG, sbp.SBP_ERR_UNSUPPORTED, sbp.SBP_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    sbp_build.build()


@pytest.mark.parametrize("kw,status", [
    (dict(dt=3), INV), (dict(table=None), INV), (dict(ids=None), INV), (dict(out=None), INV), (dict(V=0), INV), (dict(V=2 ** 31), INV),
    (dict(M=0), INV), (dict(C=0), INV), (dict(scale=float("inf")), INV), (dict(table=P + 2), INV), (dict(add=P + 8), INV), (dict(ids=P + 2), INV),
    (dict(C=12), UNS), (dict(dt=0, C=6), UNS)])
def test_forward_refusals(kw, status):
    a = dict(dt=1, table=P, V=10, C=16, ids=P, M=4, scale=1.0, add=None, out=P) | kw
    assert sbp.sbp_embedding_forward(*a.values(), stream=0, check=False) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=-1), INV), (dict(dOut=None), INV), (dict(ids=None), INV), (dict(dTable=None), INV), (dict(M_keep_cap=5), INV), (dict(M_keep_cap=-1), INV),
    (dict(keep_rows=P + 1), INV), (dict(M_keep_dev=P + 2), INV), (dict(scale=float("nan")), INV), (dict(dTable=P + 4), INV), (dict(C=20), UNS),
    (dict(workspace=None), WS), (dict(workspace=P + 128), WS), (dict(workspace_bytes=100), WS)])
def test_backward_refusals(kw, status):
    a = dict(dt=1, dOut=P, ids=P, keep_rows=P, M_keep_dev=None, M=4, M_keep_cap=4, V=10, C=16, scale=1.0, dTable=P, flags=0, workspace=P,
             workspace_bytes=1 << 30) | kw
    assert sbp.sbp_embedding_backward(*a.values(), stream=0, check=False) == status


def test_workspace_query():
    assert sbp.sbp_embedding_backward_workspace_bytes(1, 0, 0, 0) == 256
    assert sbp.sbp_embedding_backward_workspace_bytes(1, 1000, 50, 768) % 256 == 0
