"""Embedding calls and the status word: an earlier call's error leaves the outputs alone, ids of the call's own that are out of range
stop nothing but themselves."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu

ERRORS = [sbp.SBP_ERR_TIMEOUT, sbp.SBP_ERR_BAD_INDICES]
# lists that are looked through, sorted by one cluster, sorted by many blocks
ROWS = [(1, 40), (64, 40), (1000, 3000), (9000, 70), (20000, 50000), (140000, 300)]


def call(M, V, C=64, status=None, flags=0, bad=False, start=float("nan")):
    g = torch.Generator(device="cuda").manual_seed(M)
    ids = torch.randint(0, V, (M,), device="cuda", generator=g, dtype=torch.int32)
    if bad:
        ids[torch.rand(M, device="cuda", generator=g) < 0.3] = V
        ids[0] = 2 ** 31 - 1
    dOut = torch.randn((M, C), device="cuda", generator=g).bfloat16()
    nbytes = sbp.sbp_embedding_backward_workspace_bytes(1, M, V, C)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    dT = torch.full((V, C), start, device="cuda")
    sbp.sbp_embedding_backward(1, dOut, ids, None, None, M, M, V, C, 2.0, dT, flags, ws, nbytes, status)
    table, add = torch.randn((V, C), device="cuda", generator=g).bfloat16(), torch.randn((M, C), device="cuda", generator=g).bfloat16()
    outs = [dT]
    for a in (None, add):
        out = torch.full((M, C), start, dtype=torch.bfloat16, device="cuda")
        sbp.sbp_embedding_forward(1, table, V, C, ids, M, 2.0, a, out, status)
        outs.append(out)
    torch.cuda.synchronize()
    return outs


@pytest.mark.parametrize("M,V", ROWS)
@pytest.mark.parametrize("error", ERRORS)
@pytest.mark.parametrize("flags", [0, sbp.SBP_FLAG_ACCUMULATE])
@pytest.mark.parametrize("bad", [False, True])
def test_an_earlier_error_leaves_the_outputs_alone(M, V, error, flags, bad):
    status = torch.tensor([error], dtype=torch.int32, device="cuda")
    for out in call(M, V, status=status, flags=flags, bad=bad, start=5.0):
        assert (out == 5.0).all()
    assert status.item() == error


@pytest.mark.parametrize("M,V", ROWS)
def test_ids_out_of_range_stop_nothing_but_themselves(M, V):
    clean = call(M, V, bad=True)                       # without a status word
    for _ in range(5):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        for want, got in zip(clean, call_each(M, V, status)):
            assert torch.equal(want, got)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for want, got in zip(call(M, V), call(M, V, status=status)):
        assert torch.equal(want, got)
    assert status.item() == 0


def call_each(M, V, status):
    """The calls of call(), each with a word that is clear before it and holds the error behind it."""
    outs = []
    for k in range(3):
        status.zero_()
        g = torch.Generator(device="cuda").manual_seed(M)
        ids = torch.randint(0, V, (M,), device="cuda", generator=g, dtype=torch.int32)
        ids[torch.rand(M, device="cuda", generator=g) < 0.3] = V
        ids[0] = 2 ** 31 - 1
        dOut = torch.randn((M, 64), device="cuda", generator=g).bfloat16()
        table, add = torch.randn((V, 64), device="cuda", generator=g).bfloat16(), torch.randn((M, 64), device="cuda", generator=g).bfloat16()
        if k == 0:
            out = torch.full((V, 64), float("nan"), device="cuda")
            nbytes = sbp.sbp_embedding_backward_workspace_bytes(1, M, V, 64)
            ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
            sbp.sbp_embedding_backward(1, dOut, ids, None, None, M, M, V, 64, 2.0, out, 0, ws, nbytes, status)
        else:
            out = torch.full((M, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
            sbp.sbp_embedding_forward(1, table, V, 64, ids, M, 2.0, add if k == 2 else None, out, status)
        torch.cuda.synchronize()
        assert status.item() == sbp.SBP_ERR_BAD_INDICES
        outs.append(out)
    return outs


def test_behind_a_refused_norm_gradient():
    """The list of the norm's gradient is refused, its dH stays as it was, and nothing of it reaches the table's gradient."""
    M, C, V, keep = 300, 64, 30, 20
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = torch.arange(keep, dtype=torch.int32, device="cuda")
    rows[7] = 2 ** 30
    x = torch.ones((M, C), device="cuda")
    dH, dT = torch.full((M, C), 7.0, device="cuda"), torch.full((V, C), 3.0, device="cuda")
    sbp.sbp_block_norm_backward(0, 0, x, x[:keep], x[:keep], x[:keep], None, None, None, 1, 1.0, x[0], 1e-6, rows, None, M, keep, C, dH, None, None,
                                None, None, None, None, sbp.SBP_FLAG_VALIDATE, None, 0, status)
    ids = (torch.arange(M, device="cuda") % V).int()
    nbytes = sbp.sbp_embedding_backward_workspace_bytes(0, M, V, C)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    sbp.sbp_embedding_backward(0, dH, ids, None, None, M, M, V, C, 1.0, dT, sbp.SBP_FLAG_ACCUMULATE, ws, nbytes, status)
    torch.cuda.synchronize()
    assert status.item() == sbp.SBP_ERR_BAD_INDICES and (dH == 7.0).all() and (dT == 3.0).all()
