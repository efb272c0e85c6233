"""Refusals of the norm calls: every one before a launch."""
import pytest

import paper_2210_00129_b200 as sbp
from paper_2210_00129_b200 import build as sbp_build

P = 0x1000          # never dereferenced
INV, UNS, WS = sbp.SBP_ERR_INVALID_ARG, sbp.SBP_ERR_UNSUPPORTED, sbp.SBP_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    sbp_build.build()


def forward(**kw):
    a = dict(dt=1, norm=0, H=P, Y=P, post_w=P, post_b=P, gate=P, gate_group=4, residual_scale=1.0, pre_w=P, pre_b=P, eps=1e-6, M=16, C=64,
             R=P, Z=P, keep_rows=P, M_keep_dev=None, M_keep_cap=8, Y_keep=P, R_keep=P, Z_keep=P) | kw
    return sbp.sbp_block_norm_forward(*a.values(), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), INV), (dict(norm=2), INV), (dict(H=None, Y=None, post_w=None, post_b=None, gate=None, Y_keep=None), INV), (dict(M=0), INV),
    (dict(M=2 ** 31), INV), (dict(C=0), INV), (dict(M_keep_cap=17), INV), (dict(M_keep_cap=-1), INV), (dict(gate_group=0), INV),
    (dict(residual_scale=float("nan")), INV), (dict(residual_scale=1e300), INV), (dict(eps=-1.0), INV), (dict(eps=float("inf")), INV),
    (dict(eps=float("nan")), INV), (dict(C=60), UNS), (dict(C=8200), UNS), (dict(dt=0, C=62), UNS), (dict(H=P + 8), INV), (dict(Z_keep=P + 4), INV),
    (dict(keep_rows=P + 2), INV), (dict(Y=None), INV), (dict(post_w=None), INV), (dict(pre_w=None), INV), (dict(pre_w=None, pre_b=None), INV),
    (dict(pre_w=None, pre_b=None, Z=None), INV)])
def test_forward_refusals(kw, status):
    assert forward(**kw) == status


def backward(**kw):
    need = sbp.sbp_block_norm_backward_workspace_bytes(1, 16, 8, 64)
    a = dict(dt=1, norm=0, dR=P, dZ=P, R_keep=P, Y_keep=P, post_w=P, post_b=P, gate=P, gate_group=4, residual_scale=1.0, pre_w=P, eps=1e-6,
             keep_rows=P, M_keep_dev=None, M=16, M_keep_cap=8, C=64, dH=P, dY=P, dpost_w=P, dpost_b=P, dgate=P, dpre_w=P, dpre_b=P, flags=0,
             workspace=P, workspace_bytes=need) | kw
    return sbp.sbp_block_norm_backward(*a.values(), stream=0, check=False)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=7), INV), (dict(norm=-1), INV), (dict(dR=None, dZ=None, dpre_w=None, dpre_b=None), INV), (dict(R_keep=None), INV),
    (dict(pre_w=None), INV), (dict(dZ=None), INV), (dict(Y_keep=None), INV), (dict(gate=None), INV), (dict(post_w=None), INV),
    (dict(post_w=None, post_b=None), INV), (dict(Y_keep=None, dpost_w=None, dpost_b=None, dgate=None), INV), (dict(M_keep_cap=20), INV),
    (dict(flags=sbp.SBP_FLAG_VALIDATE), INV), (dict(dgate=P + 4), INV), (dict(C=8208), UNS), (dict(C=12), UNS), (dict(workspace=None), WS),
    (dict(workspace=P + 16), WS), (dict(workspace_bytes=255), WS)])
def test_backward_refusals(kw, status):
    assert backward(**kw) == status


def test_workspace_query():
    assert sbp.sbp_block_norm_backward_workspace_bytes(1, 0, 0, 0) == 256
    assert sbp.sbp_block_norm_backward_workspace_bytes(1, 100, 50, 768) % 256 == 0
