"""Norms before and after a block with its gate and residual scale, against the definition in 64 bits (gradients by autograd of
it, and by differences of it)."""
import numpy as np
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu

DT = {"bf16": (sbp.SBP_BF16, torch.bfloat16), "f32": (sbp.SBP_F32, torch.float32)}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
# A row's sums have at most 16 + 5 + 16 additions one after another (a thread's numbers, a warp's shuffles, sixteen warps), and a
# value passes through at most three such sums and some ten operations besides: 128 roundings at most.
CHAIN = 128 * 2.0 ** -24
EPS = 1e-6


def norm64(x, w, b, kind):
    x = x - x.mean(1, keepdim=True) if kind == sbp.SBP_NORM_LAYER else x
    y = x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * w
    return y if b is None else y + b


def stream64(H, Y, post_w, post_b, gate, group, scale, kind, rows):
    u = norm64(Y, post_w, post_b, kind) if post_w is not None else Y
    if gate is not None:
        u = u * gate[rows // group]
    return scale * H + u


def inputs(dtype, M, C, keep, post, bias, gate_group, mean=0.3, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000 + M + C)
    n = lambda *s, k=1.0, m=0.0: torch.randn(s, device="cuda", generator=g) * k + m
    dt = DT[dtype][1]
    rows = torch.rand(M, device="cuda", generator=g).argsort()[:keep].sort().values.int().contiguous()
    s = dict(rows=rows, H=n(M, C, k=2.0, m=mean).to(dt), Y=n(M, C, m=mean).to(dt), pre_w=n(C, k=0.2, m=1.0), pre_b=n(C) if bias else None,
             post_w=n(C, k=0.2, m=1.0) if post else None, post_b=n(C) if post and bias else None,
             gate=n((M + gate_group - 1) // gate_group, C, k=0.3, m=0.5).to(dt) if gate_group else None, group=max(gate_group, 1),
             dR=n(M, C).to(dt), dZ=n(max(keep, 1), C).to(dt), R=n(max(keep, 1), C, k=2.0, m=mean).to(dt), Yk=n(max(keep, 1), C, m=mean).to(dt))
    return s


def d(t):
    return None if t is None else t.double()


def check(name, got, want, dtype, scale, chain=CHAIN):
    """Each element within half a step of its type and the arithmetic's own error, relative to `scale`, what the row's values were made of."""
    got, want = got.double(), want.double()
    off = (got - want).abs() - HALF_STEP[dtype] * want.abs() - chain * scale
    assert not torch.isnan(got).any(), name
    assert (off <= 0).all(), (name, off.max().item(), want.abs().max().item())


def run_forward(dtype, kind, s, M, C, keep, cap=None, count=None, scale=0.9, in_place=False):
    code, dt = DT[dtype]
    cap = keep if cap is None else cap
    new = lambda r: torch.full((max(r, 1), C), float("nan"), dtype=dt, device="cuda")
    o = dict(R=s["H"].clone() if in_place else new(M), Z=new(M), Y_keep=new(cap), R_keep=new(cap), Z_keep=new(cap))
    sbp.sbp_block_norm_forward(code, kind, o["R"] if in_place else s["H"], s["Y"], s["post_w"], s["post_b"], s["gate"], s["group"], scale,
                               s["pre_w"], s["pre_b"], EPS, M, C, o["R"], o["Z"], s["rows"], count, cap, o["Y_keep"], o["R_keep"], o["Z_keep"])
    torch.cuda.synchronize()
    return o


SHAPES = [("bf16", 1, 8, 1), ("bf16", 3, 72, 2), ("bf16", 200, 256, 77), ("bf16", 37, 264, 37), ("bf16", 1500, 520, 750),
          ("bf16", 197, 768, 98), ("bf16", 64, 1024, 1), ("bf16", 33, 1032, 16), ("bf16", 130, 4096, 130), ("bf16", 9, 4104, 5),
          ("bf16", 21, 8192, 11), ("bf16", 15000, 64, 7000), ("f32", 1, 4, 1), ("f32", 50, 36, 25), ("f32", 3000, 128, 1500),
          ("f32", 65, 132, 30), ("f32", 40, 512, 40), ("f32", 41, 516, 7), ("f32", 70, 2048, 35), ("f32", 6, 4100, 3), ("f32", 5, 8192, 4)]
VARIANTS = [(0, True, True, 7), (0, False, True, 0), (1, True, False, 1), (1, False, True, 10 ** 6), (1, True, True, 0), (0, True, False, 64)]


@pytest.mark.parametrize("dtype,M,C,keep", SHAPES)
@pytest.mark.parametrize("kind,post,bias,group", VARIANTS)
def test_forward(dtype, M, C, keep, kind, post, bias, group):
    s = inputs(dtype, M, C, keep, post, bias, group)
    o = run_forward(dtype, kind, s, M, C, keep)
    every = torch.arange(M, device="cuda")
    R = stream64(d(s["H"]), d(s["Y"]), d(s["post_w"]), d(s["post_b"]), d(s["gate"]), s["group"], 0.9, kind, every)
    Z = norm64(R, d(s["pre_w"]), d(s["pre_b"]), kind)
    size = R.abs().amax(1, keepdim=True) + 4.0
    check("R", o["R"], R, dtype, size)
    # Z divides by the row's deviation: its error is the stream's over that, times the weight
    dev = ((R - R.mean(1, keepdim=True)) if kind == 0 else R).square().mean(1, keepdim=True).add(EPS).sqrt()
    check("Z", o["Z"], Z, dtype, (size / dev) * (1 + Z.abs()))
    rows = s["rows"].long()
    assert torch.equal(o["Y_keep"][:keep], s["Y"][rows])
    assert torch.equal(o["R_keep"][:keep], o["R"][rows])
    assert torch.equal(o["Z_keep"][:keep], o["Z"][rows])


def backward64(s, kind, keep, scale, with_z=True, with_r=True):
    rows = s["rows"].long()
    leaf = {n: d(s[n]).requires_grad_() for n in ("post_w", "post_b", "pre_w", "pre_b", "gate") if s[n] is not None}
    R, Y = d(s["R"])[:keep].requires_grad_(), d(s["Yk"])[:keep].requires_grad_()
    dR = d(s["dR"]) if with_r else torch.zeros_like(d(s["dR"]))
    G, out = dR[rows], {}
    if with_z:
        Z = norm64(R, leaf["pre_w"], leaf.get("pre_b"), kind)
        names = [n for n in ("pre_w", "pre_b") if n in leaf]
        g = torch.autograd.grad(Z, [R] + [leaf[n] for n in names], d(s["dZ"])[:keep])
        G = G + g[0]
        out |= {"d" + n: v for n, v in zip(names, g[1:])}
    S = stream64(torch.zeros_like(Y), Y, leaf.get("post_w"), leaf.get("post_b"), leaf.get("gate"), s["group"], scale, kind, rows)
    names = [n for n in ("post_w", "post_b", "gate") if n in leaf]
    g = torch.autograd.grad(S, [Y] + [leaf[n] for n in names], G)
    out |= {"d" + n: v for n, v in zip(names, g[1:])}
    dH = dR.clone()
    dH[rows] = G
    return {"dH": scale * dH, "dY": g[0], "G": G} | out


def run_backward(dtype, kind, s, M, C, cap, count=None, scale=0.9, flags=0, start=None, in_place=False, with_z=True, with_r=True, rows="list",
                 ws=None):
    code, dt = DT[dtype]
    o = dict(dH=s["dR"].clone() if in_place else torch.full((M, C), float("nan"), dtype=dt, device="cuda"),
             dY=torch.full((max(cap, 1), C), float("nan"), dtype=dt, device="cuda"))
    for n in ("post_w", "post_b", "pre_w", "pre_b", "gate"):
        o["d" + n] = torch.full(s[n].shape, float("nan") if start is None else start, device="cuda") if s[n] is not None else None
    if not with_z:
        o["dpre_w"] = o["dpre_b"] = None
    nbytes = sbp.sbp_block_norm_backward_workspace_bytes(code, M, cap, C)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
    sbp.sbp_block_norm_backward(code, kind, (o["dH"] if in_place else s["dR"]) if with_r else None, s["dZ"] if with_z else None, s["R"], s["Yk"],
                                s["post_w"], s["post_b"], s["gate"], s["group"], scale, s["pre_w"], EPS, s["rows"] if rows == "list" else None,
                                count, M, cap, C, o["dH"], o["dY"], o["dpost_w"], o["dpost_b"], o["dgate"], o["dpre_w"], o["dpre_b"], flags,
                                ws, nbytes)
    torch.cuda.synchronize()
    return o


def check_backward(dtype, kind, s, o, want, keep, add=0.0):
    R, Y = d(s["R"])[:keep], d(s["Yk"])[:keep]
    dev = lambda x: ((x - x.mean(1, keepdim=True)) if kind == 0 else x).square().mean(1, keepdim=True).add(EPS).sqrt()
    top = lambda x: x.abs().amax(1, keepdim=True)
    rows = s["rows"].long()
    nx, ny = top(R) / dev(R), (top(Y) / dev(Y) if s["post_w"] is not None else 1.0)
    gsize = top(d(s["dZ"])[:keep]) * 2 * nx * nx / dev(R).clamp_max(1) + 6.0          # what G was made of (weights up to 2, dR up to 6)
    size = torch.full_like(want["dH"], 6.0)
    size[rows] = size[rows] + gsize
    check("dH", o["dH"], want["dH"], dtype, size)
    ysize = gsize * 4 * (ny * ny / dev(Y).clamp_max(1) if s["post_w"] is not None else 1.0)
    check("dY", o["dY"][:keep], want["dY"], dtype, ysize)
    # a weight's gradient: terms as far off as the rows are, and sums of at most 128 additions one after another (these tests' rows
    # of a worker and of the reduction, below)
    for n in ("dpost_w", "dpost_b", "dpre_w", "dpre_b", "dgate"):
        if o[n] is None:
            continue
        terms = (top(d(s["dZ"])[:keep]) * nx if n.startswith("dpre") else gsize * 4 * (ny if s["post_w"] is not None else top(Y) + 1) + 0 * Y[:, :1])
        if n == "dgate":
            total = torch.zeros(want[n].shape[0], 1, device="cuda", dtype=torch.float64).index_add_(0, rows // s["group"], terms[:, :1])
        else:
            total = terms.sum()
        check(n, o[n], want[n] + add, "f32", total + abs(add), 2 * CHAIN)


@pytest.mark.parametrize("dtype,M,C,keep", SHAPES)
@pytest.mark.parametrize("kind,post,bias,group", VARIANTS)
def test_backward(dtype, M, C, keep, kind, post, bias, group):
    s = inputs(dtype, M, C, keep, post, bias, group)
    o = run_backward(dtype, kind, s, M, C, keep)
    check_backward(dtype, kind, s, o, backward64(s, kind, keep, 0.9), keep)


@pytest.mark.parametrize("dtype,C", [("bf16", 64), ("bf16", 776), ("f32", 516)])
def test_counts_on_the_device_accumulation_and_in_place(dtype, C):
    M, keep, cap = 300, 111, 150
    s = inputs(dtype, M, C, cap, True, True, 20)
    s["rows"][keep:] = 2 ** 31 - 1                     # behind the count: never used
    count = torch.tensor([keep], dtype=torch.int32, device="cuda")
    full = dict(s, rows=s["rows"][:keep])
    o = run_backward(dtype, 0, s, M, C, cap, count=count, flags=sbp.SBP_FLAG_ACCUMULATE, start=3.0)
    check_backward(dtype, 0, full, o, backward64(full, 0, keep, 0.9), keep, add=3.0)
    assert not o["dY"][keep:].any()
    again = run_backward(dtype, 0, s, M, C, cap, count=count, flags=sbp.SBP_FLAG_ACCUMULATE, start=3.0, in_place=True)
    for n in o:
        assert torch.equal(o[n], again[n]), n            # in place, and the same bits each time
    f = run_forward(dtype, 0, s, M, C, keep, cap=cap, count=count)
    g = run_forward(dtype, 0, s, M, C, keep, cap=cap, count=count, in_place=True)
    for n in f:
        assert torch.equal(f[n], g[n]), n
        if n.endswith("keep"):
            assert not f[n][keep:].any(), n
    # scale 1 in place: rows outside the list are not touched
    o = run_backward(dtype, 0, s, M, C, cap, count=count, scale=1.0, in_place=True)
    check_backward(dtype, 0, full, o, backward64(full, 0, keep, 1.0), keep)


@pytest.mark.parametrize("dtype,C", [("bf16", 64), ("bf16", 768), ("f32", 1032)])
@pytest.mark.parametrize("group", [1, 13, 300, 2 ** 62])
def test_entries_outside_the_tensor_are_skipped(dtype, C, group):
    M, keep = 300, 120
    s = inputs(dtype, M, C, keep, True, True, min(group, M))
    s["group"] = group
    s["rows"][:5] = torch.tensor([-2 ** 31, -7, -3, -2, -1], dtype=torch.int32)
    s["rows"][100:] = torch.arange(M, M + 20, dtype=torch.int32)
    s["rows"][-1] = 2 ** 31 - 1
    o = run_backward(dtype, 0, s, M, C, keep)
    inner = slice(5, 100)
    some = dict(s, rows=s["rows"][inner].contiguous(), dZ=s["dZ"][inner], R=s["R"][inner], Yk=s["Yk"][inner], group=min(group, M))
    want = backward64(some, 0, 95, 0.9)
    check_backward(dtype, 0, some, dict(o, dY=o["dY"][inner]), want, 95)
    assert not o["dY"][:5].any() and not o["dY"][100:].any()
    f = run_forward(dtype, 0, s, M, C, keep)
    assert torch.equal(f["R_keep"][inner], f["R"][some["rows"].long()])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_kept(dtype):
    M, C = 40, 136
    s = inputs(dtype, M, C, 10, True, True, 8)
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = run_backward(dtype, 0, s, M, C, 10, count=count)
    assert not o["dY"].any()
    for n in ("dpost_w", "dpost_b", "dpre_w", "dpre_b", "dgate"):
        assert not o[n].any(), n
    check("dH", o["dH"], 0.9 * d(s["dR"]), dtype, torch.full((M, 1), 6.0, device="cuda"))
    f = run_forward(dtype, 0, s, M, C, 0, cap=10, count=count)
    assert not f["R_keep"].any() and not f["Y_keep"].any() and not f["Z_keep"].any()
    o = run_backward(dtype, 0, s, M, C, 0)               # a capacity of none
    assert not o["dpre_w"].any() and not o["dgate"].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("with_z,with_r", [(False, True), (True, False)])
def test_missing_gradients(dtype, with_z, with_r):
    M, C, keep = 90, 200, 45
    s = inputs(dtype, M, C, keep, True, True, 30)
    o = run_backward(dtype, 1, s, M, C, keep, with_z=with_z, with_r=with_r)
    check_backward(dtype, 1, s, o, backward64(s, 1, keep, 0.9, with_z, with_r), keep)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_all_rows_without_a_list(dtype):
    M, C = 77, 264
    s = inputs(dtype, M, C, M, True, True, 10)
    want, got = run_backward(dtype, 0, s, M, C, M), run_backward(dtype, 0, s, M, C, M, rows=None)
    for n in want:
        assert torch.equal(want[n], got[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mean", [0.0, 100.0])
def test_rows_without_variance_and_rows_far_from_zero(dtype, mean):
    M, C = 12, 320
    s = inputs(dtype, M, C, M, False, True, 0, mean=mean)
    s["H"][3], s["Y"][3] = 0.0, 0.0                      # all zeros: Z is the bias
    s["H"][5], s["Y"][5] = mean + 1.0, 0.0               # one value: no variance
    o = run_forward(dtype, 0, s, M, C, M, scale=1.0)
    assert torch.equal(o["Z"][3], s["pre_b"].to(o["Z"].dtype))
    R = d(s["H"]) + d(s["Y"])
    Z = norm64(R, d(s["pre_w"]), d(s["pre_b"]), 0)
    other = [i for i in range(M) if i not in (3, 5)]
    dev = R.std(1, unbiased=False, keepdim=True)
    check("Z", o["Z"][other], Z[other], dtype, (R.abs().amax(1, keepdim=True) / dev * (1 + Z.abs()))[other])
    # the mean of one value repeated is off by a few roundings of it, and the deviation of what is left is that against sqrt(eps)
    assert (o["Z"][5].double() - d(s["pre_b"])).abs().max() <= CHAIN * (mean + 1) / EPS ** 0.5 * 2 + HALF_STEP[dtype] * 6


def test_rows_that_are_not_finite_stay_in_their_rows():
    M, C = 40, 768
    s = inputs("bf16", M, C, M, True, True, 8)
    clean = run_forward("bf16", 0, s, M, C, M)
    s["Y"][7, 5], s["H"][9, 1] = float("inf"), float("nan")
    o = run_forward("bf16", 0, s, M, C, M)
    ok = [i for i in range(M) if i not in (7, 9)]
    assert torch.equal(o["R"][ok], clean["R"][ok]) and torch.equal(o["Z"][ok], clean["Z"][ok])
    assert torch.isnan(o["Z"][7]).any() and torch.isnan(o["Z"][9]).all()


def test_parts_on_their_own():
    """A plain norm (no residual), a plain residual addition (no norms), a gate without a norm."""
    M, C = 50, 384
    s = inputs("bf16", M, C, M, True, False, 5)
    code, dt = DT["bf16"]
    new = lambda: torch.full((M, C), float("nan"), dtype=dt, device="cuda")
    Z, R = new(), new()
    sbp.sbp_block_norm_forward(code, 0, s["H"], None, None, None, None, 1, 1.0, s["pre_w"], None, EPS, M, C, None, Z)
    check("Z", Z, norm64(d(s["H"]), d(s["pre_w"]), None, 0), "bf16", torch.full((M, 1), 40.0, device="cuda"))
    sbp.sbp_block_norm_forward(code, 0, s["H"], s["Y"], None, None, s["gate"], 5, -2.0, None, None, EPS, M, C, R, None)
    want = -2.0 * d(s["H"]) + d(s["Y"]) * d(s["gate"])[torch.arange(M, device="cuda") // 5]
    check("R", R, want, "bf16", torch.full((M, 1), 30.0, device="cuda"))
    dY = new()
    sbp.sbp_block_norm_backward(code, 0, s["dR"], None, None, None, None, None, s["gate"], 5, 1.0, None, EPS, None, None, M, M, C, None, dY, None,
                                None, None, None, None, 0, None, 0)
    check("dY", dY, d(s["dR"]) * d(s["gate"])[torch.arange(M, device="cuda") // 5], "bf16", torch.full((M, 1), 6.0, device="cuda"))


def test_gradient_against_differences():
    """d/dt of sum(dZ Z + dR R) along a direction in H and Y, by central differences of the forward in 64 bits."""
    M, C, kind = 6, 40, 0
    s = inputs("f32", M, C, M, True, True, 2)
    s["rows"] = torch.arange(M, dtype=torch.int32, device="cuda")
    every = torch.arange(M, device="cuda")

    def loss(H, Y):
        R = stream64(H, Y, d(s["post_w"]), d(s["post_b"]), d(s["gate"]), s["group"], 0.9, kind, every)
        return (d(s["dZ"]) * norm64(R, d(s["pre_w"]), d(s["pre_b"]), kind) + d(s["dR"]) * R).sum()

    f = run_forward("f32", kind, s, M, C, M)
    s["R"], s["Yk"] = f["R_keep"], f["Y_keep"]
    o = run_backward("f32", kind, s, M, C, M)
    g = torch.Generator(device="cuda").manual_seed(4)
    for _ in range(4):
        vH, vY = (torch.randn((M, C), device="cuda", generator=g, dtype=torch.float64) for _ in range(2))
        h = 1e-5
        num = (loss(d(s["H"]) + h * vH, d(s["Y"]) + h * vY) - loss(d(s["H"]) - h * vH, d(s["Y"]) - h * vY)) / (2 * h)
        got = (d(o["dH"]) * vH + d(o["dY"]) * vY).sum()
        # R is rounded to fp32 between the two (2^-24), the gradients are fp32, and the differences are off by h^2
        assert abs(got - num) <= 1e-5 * (d(o["dH"]).norm() * vH.norm() + d(o["dY"]).norm() * vY.norm())


def test_streams_graphs_and_one_workspace_a_call():
    M, C, keep = 600, 512, 300
    s = inputs("bf16", M, C, keep, True, True, 100)
    want = run_backward("bf16", 0, s, M, C, keep)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run_backward("bf16", 0, s, M, C, keep)
        for n in want:
            assert torch.equal(want[n], got[n]), n
        nbytes = sbp.sbp_block_norm_backward_workspace_bytes(1, M, keep, C)
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        o = {n: torch.full_like(v, float("nan")) for n, v in want.items()}
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            sbp.sbp_block_norm_backward(1, 0, s["dR"], s["dZ"], s["R"], s["Yk"], s["post_w"], s["post_b"], s["gate"], s["group"], 0.9, s["pre_w"],
                                        EPS, s["rows"], None, M, keep, C, o["dH"], o["dY"], o["dpost_w"], o["dpost_b"], o["dgate"], o["dpre_w"],
                                        o["dpre_b"], 0, ws, nbytes)
        for _ in range(2):
            for v in o.values():
                v.fill_(float("nan"))
            graph.replay()
            side.synchronize()
            for n in want:
                assert torch.equal(want[n], o[n]), n


def test_a_bad_list_is_reported_and_nothing_is_written():
    M, C, keep = 100, 256, 20
    s = inputs("bf16", M, C, keep, True, True, 10)
    s["rows"][7] = 2 ** 30
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dY = torch.full((keep, C), 5.0, dtype=torch.bfloat16, device="cuda")
    sbp.sbp_block_norm_backward(1, 0, s["dR"], s["dZ"], s["R"], s["Yk"], s["post_w"], s["post_b"], None, 1, 1.0, s["pre_w"], EPS, s["rows"], None, M,
                                keep, C, None, dY, None, None, None, None, None, sbp.SBP_FLAG_VALIDATE, None, 0, status)
    torch.cuda.synchronize()
    assert status.item() == sbp.SBP_ERR_BAD_INDICES and (dY == 5.0).all()
