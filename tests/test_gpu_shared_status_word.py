"""Calls on one stream while the status word they were given changes on another: every call ends, and those that begin and end with
a clear word are right."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu


def norm_calls(status):
    """Rows of three warps, of sixteen, and several rows a warp; forward and backward with all sums."""
    calls = []
    for dtype, code, C in ((torch.bfloat16, 1, 768), (torch.bfloat16, 1, 8192), (torch.float32, 0, 2048), (torch.float32, 0, 64)):
        M, keep = 700, 350
        g = torch.Generator(device="cuda").manual_seed(C)
        n = lambda *s: torch.randn(s, device="cuda", generator=g)
        H, Y, R, Z, dH = (n(M, C).to(dtype) for _ in range(5))
        Yk, Rk, Zk, dZ, dY = (n(keep, C).to(dtype) for _ in range(5))
        rows = torch.arange(0, M, 2, dtype=torch.int32, device="cuda")
        gate, w, b = n(M // 70, C).to(dtype), n(C), n(C)
        sums = [torch.empty(C, device="cuda") for _ in range(4)] + [torch.empty(M // 70, C, device="cuda")]
        nbytes = sbp.sbp_block_norm_backward_workspace_bytes(code, M, keep, C)
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        calls.append((lambda a=(code, 0, H, Y, w, b, gate, 70, 0.9, w, b, 1e-6, M, C, R, Z, rows, None, keep, Yk, Rk, Zk, status):
                      sbp.sbp_block_norm_forward(*a), [R, Z, Yk, Rk, Zk]))
        kept = (n(keep, C).to(dtype), n(keep, C).to(dtype))
        calls.append((lambda a=(code, 0, H, dZ, *kept, w, b, gate, 70, 0.9, w, 1e-6, rows, None, M, keep, C, dH, dY, sums[0], sums[1], sums[4],
                                sums[2], sums[3], 0, ws, nbytes, status): sbp.sbp_block_norm_backward(*a), [dH, dY] + sums))
    return calls


def ortho_calls(status):
    calls = []
    for code, count, rows, cols in ((1, 2, 300, 400), (0, 1, 260, 200), (1, 1, 100, 257), (1, 3, 64, 1000)):
        G = torch.randn((count, rows, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(rows))
        O = torch.empty(G.shape, dtype=torch.bfloat16 if code else torch.float32, device="cuda")
        nbytes = sbp.sbp_orthogonalize_workspace_bytes(code, count, rows, cols)
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        calls.append((lambda a=(code, G, None, 0.0, count, rows, cols, 3, 1e-7, 1.0, O, 0, ws, nbytes, status): sbp.sbp_orthogonalize(*a), [O]))
    return calls


@pytest.mark.parametrize("make", [norm_calls, ortho_calls])
def test_a_word_that_changes_meanwhile(make):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = make(status)
    want = []
    for call, outs in calls:
        call()
        want.append([o.clone() for o in outs])
    torch.cuda.synchronize()
    assert status.item() == 0
    work, other = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(60):
        with torch.cuda.stream(work):
            for call, _ in calls:
                call()
        with torch.cuda.stream(other):
            for _ in range(2 * len(calls)):
                status.fill_(sbp.SBP_ERR_BAD_INDICES)
                status.zero_()
    torch.cuda.synchronize()
    status.zero_()
    for (call, outs), w in zip(calls, want):
        for o in outs:
            o.fill_(float("nan"))
        call()
        torch.cuda.synchronize()
        assert status.item() == 0
        for o, x in zip(outs, w):
            assert torch.equal(o, x)
