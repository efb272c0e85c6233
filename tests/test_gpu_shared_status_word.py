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


def layer_calls(status):
    """Layers on the tensor cores (wide and narrow tiles, pairs of blocks), in fp32 both ways, and attention."""
    calls = []
    new = lambda *s, dtype=torch.bfloat16: torch.randn(s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(len(calls))).to(dtype)
    for dtype, code, M, C_in, C_out, flags in ((torch.bfloat16, 1, 12544, 768, 2304, 0), (torch.bfloat16, 1, 2000, 96, 384, 0),
                                               (torch.bfloat16, 1, 2000, 64, 64, sbp.SBP_FLAG_W_OUT_IN), (torch.float32, 0, 2000, 768, 768, 0),
                                               (torch.float32, 0, 2000, 64, 64, sbp.SBP_FLAG_PLAIN_FMA)):
        keep = M // 2
        rows = torch.arange(0, M, 2, dtype=torch.int32, device="cuda")
        X, dY, W = new(M, C_in, dtype=dtype), new(M, C_out, dtype=dtype), new(C_in, C_out, dtype=dtype)
        Xk, dX, Y = new(keep, C_in, dtype=dtype), new(M, C_in, dtype=dtype), new(M, C_out, dtype=dtype)
        dW, db, bias = torch.empty(C_in, C_out, device="cuda"), torch.empty(C_out, device="cuda"), new(C_out, dtype=torch.float32)
        nbytes = sbp.sbp_linear_backward_workspace_bytes(code, M, keep, C_in, C_out)
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        calls.append((lambda a=(code, X, W, bias, M, C_in, C_out, Y, None, None, 0, None, flags, status): sbp.sbp_linear_forward(*a), [Y]))
        calls.append((lambda a=(code, Xk, dY, W, rows, None, M, keep, C_in, C_out, dW, db, dX, flags, ws, nbytes, status):
                      sbp.sbp_linear_backward(*a), [dW, db, dX]))
    B, N, heads = 8, 196, 4
    Q, K, V, dA, dQ, dK, dV = (new(B * N, heads * 64) for _ in range(7))
    offs = torch.arange(0, B * 98 + 1, 98, dtype=torch.int32, device="cuda")
    tokens = torch.arange(0, B * N, 2, dtype=torch.int32, device="cuda")
    calls.append((lambda a=(1, Q, K, V, heads * 64, dA, heads * 64, tokens, offs, tokens, offs, B, N, heads, 64, 98, dQ, dK, dV, heads * 64, 0,
                            status): sbp.sbp_attention_backward(*a), [dQ, dK, dV]))
    return calls


# (warps of a layer's block that see the word change between them end at their waits' limit of two seconds: few rounds)
@pytest.mark.parametrize("make,rounds,flips", [(norm_calls, 60, 30), (ortho_calls, 60, 30), (layer_calls, 3, 1)])
def test_a_word_that_changes_meanwhile(make, rounds, flips):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = make(status)
    want = []
    for call, outs in calls:
        call()
        want.append([o.clone() for o in outs])
    torch.cuda.synchronize()
    assert status.item() == 0
    work, other = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(rounds):
        with torch.cuda.stream(work):
            for call, _ in calls:
                call()
        with torch.cuda.stream(other):
            for _ in range(flips):
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
