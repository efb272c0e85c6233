"""Rows of a table by id and the table's gradient, against sums in 64 bits."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu

DT = {"bf16": (sbp.SBP_BF16, torch.bfloat16, 2.0 ** -8), "f32": (sbp.SBP_F32, torch.float32, 2.0 ** -24)}


def ids_of(how, M, V, g):
    if how == "one":
        ids = torch.full((M,), V - 1, device="cuda")
    elif how == "position":
        ids = torch.arange(M, device="cuda") % V
    elif how == "skewed":
        ids = (torch.rand(M, device="cuda", generator=g) ** 6 * V).long()
    else:
        ids = torch.randint(0, V, (M,), device="cuda", generator=g)
    return ids.int()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,C", [(1, 1, 8), (7, 3, 40), (500, 50257, 768), (1025, 100, 1032), (3, 5, 12288)])
@pytest.mark.parametrize("with_add", [False, True])
def test_forward(dtype, M, V, C, with_add):
    code, dt, half = DT[dtype]
    g = torch.Generator(device="cuda").manual_seed(M + C)
    table = torch.randn((V, C), device="cuda", generator=g).to(dt)
    add = torch.randn((M, C), device="cuda", generator=g).to(dt) if with_add else None
    ids = ids_of("uniform", M, V, g)
    if M > 1:
        ids[M // 2] = -1
        ids[M - 1] = V - 1
    out = torch.full((M, C), float("nan"), dtype=dt, device="cuda")
    sbp.sbp_embedding_forward(code, table, V, C, ids, M, 27.75, add, out)
    rows = table.double()[ids.long().clamp_min(0)] * 27.75
    rows[ids < 0] = 0
    want = rows + add.double() if with_add else rows
    # one fused multiply-add and one rounding to the type
    assert ((out.double() - want).abs() <= half * want.abs() * 1.01 + 2.0 ** -24 * want.abs()).all()
    if with_add:
        same = add.clone()
        sbp.sbp_embedding_forward(code, table, V, C, ids, M, 27.75, same, same)
        assert torch.equal(same, out)


def gradient(dtype, dOut, ids, rows, M, cap, V, C, scale=3.0, flags=0, start=float("nan"), count=None, status=None):
    nbytes = sbp.sbp_embedding_backward_workspace_bytes(DT[dtype][0], cap, V, C)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    dT = torch.full((V, C), start, device="cuda")
    sbp.sbp_embedding_backward(DT[dtype][0], dOut, ids, rows, count, M, cap, V, C, scale, dT, flags, ws, nbytes, status)
    torch.cuda.synchronize()
    return dT


def check(dT, dOut, ids, rows, V, scale=3.0, start=0.0):
    """dOut: the gradients of `rows`, one each.  Every sum has one rounding an addition and one for the scale; a sum of k rows
    in pieces has k additions or fewer one after another."""
    k = ids.long()[rows]
    ok = (k >= 0) & (k < V)
    k, x = k[ok], dOut.double()[ok]
    want = torch.zeros(dT.shape, dtype=torch.float64, device="cuda").index_add_(0, k, x) * scale
    size = torch.zeros_like(want).index_add_(0, k, x.abs()) * scale
    n = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, k, torch.ones_like(k, dtype=torch.float64))
    depth = n.clamp_max(1500)[:, None] + 3             # (no piece of these tests has over 1024 places; the pieces are joined in eights)
    assert ((dT.double() - start - want).abs() <= depth * 2.0 ** -24 * (size + abs(start))).all()
    assert (dT[n == 0] == start).all()


SHAPES = [(1, 1, 8, "one"), (5, 1, 8, "one"), (31, 7, 72, "uniform"), (4096, 300, 256, "skewed"), (4097, 255, 264, "uniform"), (5000, 256, 64, "position"),
          (12544, 196, 768, "position"), (20000, 50257, 136, "skewed"), (9000, 1, 512, "one"), (70000, 70000, 8, "uniform"), (600000, 1000, 16, "skewed"),
          (33, 1 << 20, 8, "uniform"), (8192, 5, 1032, "uniform"), (6, 17, 8192, "uniform")]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,V,C,how", SHAPES)
def test_gradient(dtype, M, V, C, how):
    g = torch.Generator(device="cuda").manual_seed(M)
    ids = ids_of(how, M, V, g)
    ids[torch.rand(M, device="cuda", generator=g) < 0.02] = -3
    dOut = torch.randn((M, C), device="cuda", generator=g).to(DT[dtype][1])
    keep = (M + 1) // 2
    rows = torch.rand(M, device="cuda", generator=g).argsort()[:keep].sort().values
    r32 = rows.int().contiguous()
    dT = gradient(dtype, dOut, ids, r32, M, keep, V, C)
    check(dT, dOut[rows], ids, rows, V)
    assert torch.equal(dT, gradient(dtype, dOut, ids, r32, M, keep, V, C))
    packed = dOut[rows].contiguous()
    assert torch.equal(dT, gradient(dtype, packed, ids, r32, M, keep, V, C, flags=sbp.SBP_FLAG_DY_COMPACT))
    more = gradient(dtype, dOut, ids, r32, M, keep, V, C, flags=sbp.SBP_FLAG_ACCUMULATE, start=2.0)
    check(more, dOut[rows], ids, rows, V, start=2.0)
    every = torch.arange(M, device="cuda")
    check(gradient(dtype, dOut, ids, None, M, M, V, C), dOut, ids, every, V)


@pytest.mark.parametrize("M", [300, 9000])
def test_count_on_the_device_and_lists_in_any_order(M):
    V, C, cap, keep = 50, 128, M, M // 3
    g = torch.Generator(device="cuda").manual_seed(1)
    ids, dOut = ids_of("uniform", M, V, g), torch.randn((M, C), device="cuda", generator=g)
    rows = torch.rand(M, device="cuda", generator=g).argsort()
    r32 = rows.int().contiguous()
    r32[keep:] = 2 ** 31 - 1                           # behind the count: never used
    for n in (keep, 1, 0):
        count = torch.tensor([n], dtype=torch.int32, device="cuda")
        check(gradient("f32", dOut, ids, r32, M, cap, V, C, count=count), dOut[rows[:n]], ids, rows[:n], V)
    assert not gradient("f32", dOut, ids, r32, M, 0, V, C).any()
    twice = torch.cat([r32[:keep], r32[:keep]]).contiguous()              # a row listed twice counts twice
    check(gradient("f32", dOut, ids, twice, M, 2 * keep, V, C), torch.cat([dOut[rows[:keep]]] * 2), ids, torch.cat([rows[:keep]] * 2), V)


@pytest.mark.parametrize("M", [64, 9000])
def test_ids_and_rows_out_of_range(M):
    V, C = 30, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    ids, dOut = ids_of("uniform", M, V, g), torch.randn((M, C), device="cuda", generator=g)
    ids[3], ids[M - 1], ids[9] = V, 2 ** 31 - 1, -2 ** 31
    rows = torch.arange(M, device="cuda", dtype=torch.int32)
    rows[20], rows[21] = -5, M                         # skipped
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dT = gradient("f32", dOut, ids, rows, M, M, V, C, status=status)
    assert status.item() == sbp.SBP_ERR_BAD_INDICES
    ok = torch.tensor([i for i in range(M) if i not in (3, M - 1, 9, 20, 21)], device="cuda")
    check(dT, dOut[ok], ids, ok, V)
    table, out = torch.randn((V, C), device="cuda", generator=g), torch.full((M, C), float("nan"), device="cuda")
    status.zero_()
    sbp.sbp_embedding_forward(0, table, V, C, ids, M, 1.0, None, out, status)
    torch.cuda.synchronize()
    assert status.item() == sbp.SBP_ERR_BAD_INDICES
    assert not out[[3, M - 1, 9]].any() and torch.equal(out[ok], table[ids.long()[ok]])


def test_gradients_that_are_not_finite_stay_with_their_ids():
    M, V, C = 400, 20, 64
    ids = (torch.arange(M, device="cuda") % V).int()
    dOut = torch.ones((M, C), dtype=torch.bfloat16, device="cuda")
    dOut[25, 3], dOut[47, 5] = float("nan"), float("inf")
    dT = gradient("bf16", dOut, ids, None, M, M, V, C, scale=1.0)
    want = torch.full((V, C), 20.0, device="cuda")
    want[5, 3], want[7, 5] = float("nan"), float("inf")
    assert torch.equal(torch.nan_to_num(dT, 1e9, 1e8), torch.nan_to_num(want, 1e9, 1e8))


def test_captured_and_replayed_on_another_stream():
    M, V, C = 6000, 900, 256
    g = torch.Generator(device="cuda").manual_seed(3)
    ids, dOut = ids_of("skewed", M, V, g), torch.randn((M, C), device="cuda", generator=g).bfloat16()
    want = gradient("bf16", dOut, ids, None, M, M, V, C)
    nbytes = sbp.sbp_embedding_backward_workspace_bytes(1, M, V, C)
    ws, dT = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.empty((V, C), device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sbp.sbp_embedding_backward(1, dOut, ids, None, None, M, M, V, C, 3.0, dT, 0, ws, nbytes)
    for _ in range(2):
        dT.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dT, want)


@pytest.mark.parametrize("M", [700, 9000])
def test_calls_at_once_on_three_streams(M):
    V, C = 5000, 256
    g = torch.Generator(device="cuda").manual_seed(4)
    ids = [ids_of(how, M, V, g) for how in ("skewed", "uniform", "one")]
    dOut = torch.randn((M, C), device="cuda", generator=g).bfloat16()
    want = [gradient("bf16", dOut, i, None, M, M, V, C) for i in ids]
    nbytes = sbp.sbp_embedding_backward_workspace_bytes(1, M, V, C)
    ws = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in ids]
    dT = [torch.full_like(w, float("nan")) for w in want]
    streams = [torch.cuda.Stream() for _ in ids]
    torch.cuda.synchronize()
    for _ in range(4):
        for i, w, t, s in zip(ids, ws, dT, streams):
            with torch.cuda.stream(s):
                sbp.sbp_embedding_backward(1, dOut, i, None, None, M, M, V, C, 3.0, t, 0, w, nbytes)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(dT, want))
