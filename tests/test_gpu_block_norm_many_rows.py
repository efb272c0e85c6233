"""The norm kernels where their loops go round: several rows of a worker, lane groups of a warp that change gate row at different times,
gate rows inside a worker's rows, workers with entries inside and outside the tensor; chunks of several rows forward.  Gradients
of weights are held to the bounds of norm_bounds.py, which a single kept row left out breaks."""
import pytest
import torch

import norm_bounds
import paper_2210_00129_b200 as sbp
import test_gpu_block_norm as base

pytestmark = pytest.mark.gpu

# rows of a worker behind: one to four or more at each shape of a worker
MANY = [("bf16", 60000, 64, 30000), ("f32", 40000, 64, 39000), ("f32", 40000, 128, 20000), ("bf16", 30000, 128, 30000), ("bf16", 15000, 256, 14000),
        ("f32", 9000, 200, 8000), ("bf16", 4000, 512, 3900), ("bf16", 3500, 768, 3400), ("f32", 2500, 1000, 2400), ("bf16", 1700, 2048, 1600),
        ("f32", 1200, 4096, 1100), ("bf16", 900, 8192, 800)]
KINDS = [(0, True, True), (1, False, True), (0, True, False)]


def exact(s, rows, kind, with_z=True):
    d = lambda t: None if t is None else t.double()
    kept = {n: d(s[n]) for n in ("pre_w", "post_w", "post_b", "gate")} | {n: d(s[n])[:rows.numel()] for n in ("R", "Yk", "dZ")}
    return norm_bounds.backward(kept | dict(group=s["group"]), kind, rows, d(s["dR"])[rows], with_z)


@pytest.mark.parametrize("dtype,M,C,keep", MANY)
@pytest.mark.parametrize("kind,post,bias", KINDS)
@pytest.mark.parametrize("group", [0, 1, 3, 7, 64, 10 ** 6])
def test_backward(dtype, M, C, keep, kind, post, bias, group):
    s = base.inputs(dtype, M, C, keep, post, bias, group)
    o = base.run_backward(dtype, kind, s, M, C, keep)
    base.check_backward(dtype, kind, s, o, base.backward64(s, kind, keep, 0.9), keep)
    want = exact(s, s["rows"].long(), kind)
    norm_bounds.check(o, want)
    more = base.run_backward(dtype, kind, s, M, C, keep, flags=sbp.SBP_FLAG_ACCUMULATE, start=3.0)
    norm_bounds.check(more, want, add=3.0)
    for n in ("dH", "dY"):
        assert torch.equal(o[n], more[n]), n


@pytest.mark.parametrize("dtype,M,C,keep", base.SHAPES)
@pytest.mark.parametrize("kind,post,bias,group", base.VARIANTS)
def test_weight_gradients_of_the_other_shapes(dtype, M, C, keep, kind, post, bias, group):
    s = base.inputs(dtype, M, C, keep, post, bias, group)
    norm_bounds.check(base.run_backward(dtype, kind, s, M, C, keep), exact(s, s["rows"].long(), kind))


@pytest.mark.parametrize("dtype,M,C,keep", MANY)
@pytest.mark.parametrize("group", [1, 7, 500, 2 ** 62])
def test_entries_outside_the_tensor_among_a_workers_rows(dtype, M, C, keep, group):
    s = base.inputs(dtype, M, C, keep, True, True, min(group, M))
    s["group"] = group
    before, behind = 3 + keep // 7, 5 + keep // 9      # whole workers', and parts of one's
    s["rows"][:before] = torch.arange(-before, 0, device="cuda", dtype=torch.int32) - 2 ** 30
    s["rows"][keep - behind:] = torch.arange(behind, device="cuda", dtype=torch.int32) + M
    inner = slice(before, keep - behind)
    o = base.run_backward(dtype, 0, s, M, C, keep)
    some = dict(s, rows=s["rows"][inner].contiguous(), dZ=s["dZ"][inner], R=s["R"][inner], Yk=s["Yk"][inner], group=min(group, M))
    count = keep - before - behind
    base.check_backward(dtype, 0, some, dict(o, dY=o["dY"][inner]), base.backward64(some, 0, count, 0.9), count)
    norm_bounds.check(o, exact(some, some["rows"].long(), 0))
    assert not o["dY"][:before].any() and not o["dY"][keep - behind:].any()


@pytest.mark.parametrize("dtype,M,C,keep", [("bf16", 60000, 64, 30000), ("f32", 60000, 64, 59999), ("f32", 40000, 128, 20000), ("bf16", 114000, 128, 1000),
                                            ("bf16", 15000, 256, 7000), ("f32", 57000, 200, 57000), ("bf16", 2500, 768, 1000), ("f32", 2400, 1032, 2000)])
@pytest.mark.parametrize("kind,post,bias,group", base.VARIANTS)
def test_forward_chunks_of_several_rows(dtype, M, C, keep, kind, post, bias, group):
    base.test_forward(dtype, M, C, keep, kind, post, bias, group)


def test_calls_at_once_on_three_streams():
    shapes = [("bf16", 6000, 768, 3000), ("f32", 9000, 128, 4500), ("bf16", 1500, 4096, 1500)]
    made = [base.inputs(d, M, C, keep, True, True, 50) for d, M, C, keep in shapes]
    fwd = [base.run_forward(d, 0, s, M, C, keep) for s, (d, M, C, keep) in zip(made, shapes)]
    bwd = [base.run_backward(d, 0, s, M, C, keep) for s, (d, M, C, keep) in zip(made, shapes)]
    streams = [torch.cuda.Stream() for _ in shapes]
    outs, spaces = [], []
    for s, f, o, (d, M, C, keep) in zip(made, fwd, bwd, shapes):
        outs.append({n: torch.full_like(t, float("nan")) for n, t in (f | o).items()})
        spaces.append(torch.empty(sbp.sbp_block_norm_backward_workspace_bytes(base.DT[d][0], M, keep, C), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(4):
        for s, o, ws, stream, (d, M, C, keep) in zip(made, outs, spaces, streams, shapes):
            code = base.DT[d][0]
            with torch.cuda.stream(stream):
                sbp.sbp_block_norm_forward(code, 0, s["H"], s["Y"], s["post_w"], s["post_b"], s["gate"], s["group"], 0.9, s["pre_w"], s["pre_b"],
                                           base.EPS, M, C, o["R"], o["Z"], s["rows"], None, keep, o["Y_keep"], o["R_keep"], o["Z_keep"])
                sbp.sbp_block_norm_backward(code, 0, s["dR"], s["dZ"], s["R"], s["Yk"], s["post_w"], s["post_b"], s["gate"], s["group"], 0.9,
                                            s["pre_w"], base.EPS, s["rows"], None, M, keep, C, o["dH"], o["dY"], o["dpost_w"], o["dpost_b"],
                                            o["dgate"], o["dpre_w"], o["dpre_b"], 0, ws, ws.numel())
    torch.cuda.synchronize()
    for o, f, b in zip(outs, fwd, bwd):
        for n, want in (f | b).items():
            assert torch.equal(o[n], want), n
