"""Refusals of sbp_orthogonalize: every one before a launch."""
import pytest

import paper_2210_00129_b200 as sbp
from paper_2210_00129_b200 import build as sbp_build

P = 0x1000          # never dereferenced
INV, UNS, WS = sbp.SBP_ERR_INVALID_ARG, sbp.SBP_ERR_UNSUPPORTED, sbp.SBP_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    sbp_build.build()


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), INV), (dict(G=None), INV), (dict(O=None), INV), (dict(G=P + 4), INV), (dict(momentum=P + 8), INV), (dict(O=P + 2), INV),
    (dict(count=0), INV), (dict(rows=0), INV), (dict(cols=-1), INV), (dict(steps=0), INV), (dict(steps=33), INV), (dict(beta=float("nan")), INV),
    (dict(eps=-1e-9), INV), (dict(eps=float("inf")), INV), (dict(scale=1e300), INV), (dict(momentum=None, flags=sbp.SBP_FLAG_NESTEROV), INV),
    (dict(rows=2 ** 17), UNS), (dict(cols=2 ** 17), UNS), (dict(count=2 ** 16), UNS), (dict(workspace=None), WS), (dict(workspace=P + 16), WS),
    (dict(workspace_bytes=255), WS), (dict(rows=640, cols=320, workspace_bytes=1000), WS)])
def test_refusals(kw, status):
    a = dict(dt=1, G=P, momentum=P, beta=0.9, count=2, rows=64, cols=32, steps=5, eps=1e-7, scale=1.0, O=P, flags=0, workspace=P,
             workspace_bytes=1 << 30) | kw
    assert sbp.sbp_orthogonalize(*a.values(), stream=0, check=False) == status


def test_workspace_query():
    q = sbp.sbp_orthogonalize_workspace_bytes
    assert q(1, 0, 0, 0) == 256 and q(1, 2 ** 16, 8, 8) == 256
    assert q(1, 3, 768, 768) % 256 == 0 and q(0, 3, 768, 768) > q(1, 3, 768, 768)
