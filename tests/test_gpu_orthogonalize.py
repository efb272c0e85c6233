"""Newton-Schulz orthogonalisation against the iteration in 64 bits, and against the same with the documented roundings.

Tolerances: the library's own for its two types, a relative Frobenius error of 5e-3 (bf16) and 1e-5 (fp32).  Beside that the error
may be twice that of the iteration in 64 bits with the kernel's roundings (its values lie elsewhere only where a sum fell on the
other side of a border) and half a step of the output type, and no element may be off by over 0.1 (bf16) or 1e-3 (fp32) rms
beside its own rounding: a row left out of a product moves whole rows by more."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu

DT = {"bf16": (sbp.SBP_BF16, torch.bfloat16, 2.0 ** -8), "f32": (sbp.SBP_F32, torch.float32, 2.0 ** -24)}
NS = (3.4445, -4.7750, 2.0315)


def first(x):
    return (x * 4096).half().double() / 4096


def both(x):
    f = first(x)
    return f + first(x - f)


def iterate(U, steps, eps, rounded=None):
    """The iteration in 64 bits; rounded: "fast" or "exact", the roundings of the two kernels."""
    a, b, c = NS
    tall = U.shape[1] > U.shape[2]
    X = U.double().mT if tall else U.double()
    X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + eps)
    eye = torch.eye(X.shape[1], device="cuda", dtype=torch.float64)
    for _ in range(steps):
        if rounded is None:
            A = X @ X.mT
            X = a * X + (b * A + c * (A @ A)) @ X
            continue
        X = both(X)
        lo = (lambda m: m - first(m)) if rounded == "exact" else torch.zeros_like
        hold = both if rounded == "exact" else first
        mul = lambda p, q: first(p) @ first(q) + lo(p) @ first(q) + first(p) @ lo(q)
        A = mul(X, X.mT)
        d = A * eye
        A = hold(A)
        B = b * A + c * mul(A, A)
        B = B + (b * (d - A * eye) + c * (d * d - (A * eye) ** 2))
        f = (a + (B * eye).sum(2))[:, :, None]
        X = f * X + mul(hold(B - B * eye), X)
    return X.mT if tall else X


def gradient(how, count, rows, cols):
    g = torch.Generator(device="cuda").manual_seed(rows * 1000 + cols)
    n = lambda *s: torch.randn(s, device="cuda", generator=g)
    G = n(count, rows, cols)
    if how == "low":                                   # rank at most 20, over a little noise
        k = min(20, rows, cols)
        G = n(count, rows, k) @ n(count, k, cols) + 0.01 * G
    elif how == "mean":
        G = G + 3
    elif how == "rows":                                # rows of very different sizes
        G = G * torch.logspace(0, -4, rows, device="cuda")[:, None]
    return G


def run(dtype, G, steps=5, momentum=None, beta=0.9, nesterov=False, eps=1e-7, scale=1.0, status=None):
    count, rows, cols = G.shape
    O = torch.full(G.shape, float("nan"), dtype=DT[dtype][1], device="cuda")
    nbytes = sbp.sbp_orthogonalize_workspace_bytes(DT[dtype][0], count, rows, cols)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")           # NaN wherever it is read before it is written
    sbp.sbp_orthogonalize(DT[dtype][0], G, momentum, beta, count, rows, cols, steps, eps, scale, O, sbp.SBP_FLAG_NESTEROV if nesterov else 0, ws,
                          nbytes, status)
    torch.cuda.synchronize()
    return O


def check(dtype, O, U, steps=5, eps=1e-7, scale=1.0):
    want = iterate(U, steps, eps)
    exact = dtype == "f32" or min(U.shape[1:]) <= 128
    rounded = iterate(U, steps, eps, "exact" if exact else "fast")
    norm = lambda x: x.square().sum((1, 2)).sqrt()
    half = DT[dtype][2]
    off, size, model = norm(O.double() / scale - want), norm(want), norm(rounded - want)
    assert torch.isfinite(O).all()
    assert (off <= 2 * model + half * size + (1e-5 * size if exact else 0)).all(), (off / size, model / size)
    assert (off <= {"bf16": 5e-3, "f32": 1e-5}[dtype] * size + 2 * (model if dtype == "f32" else 0 * model)).all(), off / size
    rms = (size / (U.shape[1] * U.shape[2]) ** 0.5)[:, None, None]
    assert ((O.double() / scale - want).abs() <= half * 1.01 * want.abs() + {"bf16": 0.1, "f32": 1e-3}[dtype] * rms).all()


SIZES = [(1, 1, 1), (1, 1, 100), (2, 100, 1), (3, 8, 8), (2, 5, 13), (1, 64, 64), (1, 100, 257), (2, 128, 128), (1, 129, 200), (2, 136, 136),
         (1, 256, 512), (1, 512, 256), (1, 300, 300), (2, 200, 1000), (1, 1000, 136), (1, 768, 768), (3, 384, 640), (1, 2304, 768), (40, 130, 140),
         (1, 131, 4099), (1, 128, 2048), (2, 2048, 128), (1, 100, 513), (3, 64, 1000), (1, 17, 129), (1, 260, 60), (2, 3, 1500), (1, 128, 2049),
         (1, 2100, 24), (200, 40, 300), (1, 520, 2100), (2, 1500, 260), (1, 3000, 140),
         (28, 500, 440), (30, 440, 500), (57, 264, 300)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count,rows,cols", SIZES)
@pytest.mark.parametrize("how", ["normal", "low"])
def test_against_the_iteration(dtype, count, rows, cols, how):
    G = gradient(how, count, rows, cols)
    O = run(dtype, G)
    check(dtype, O, G)
    assert torch.equal(O, run(dtype, G))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("how", ["mean", "rows"])
@pytest.mark.parametrize("rows,cols", [(192, 320), (320, 192), (100, 100)])
def test_other_gradients(dtype, how, rows, cols):
    G = gradient(how, 2, rows, cols)
    check(dtype, run(dtype, G), G)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("steps", [1, 2, 9])
def test_steps_and_scale(dtype, steps):
    G = gradient("normal", 1, 160, 224)
    check(dtype, run(dtype, G, steps=steps, scale=-0.5), G, steps=steps, scale=-0.5)


def test_singular_values_come_near_one():
    for shape in ((1, 256, 256), (1, 200, 600), (1, 600, 200)):
        s = torch.linalg.svdvals(run("f32", gradient("normal", *shape)).double())
        assert s.max() < 1.25 and s.median() > 0.65      # what the quintic gives for values above a ^ -5


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e18, 1e33])
def test_gradients_of_any_size(size):
    G = gradient("normal", 1, 144, 200)
    O, P = run("bf16", G, eps=0.0), run("bf16", G * size, eps=0.0)
    check("bf16", P, G * size, eps=0.0)
    assert (O.double() - P.double()).abs().max() <= 0.02


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(200, 136), (33, 67)])
@pytest.mark.parametrize("nesterov", [False, True])
def test_momentum(dtype, rows, cols, nesterov):
    G, M = gradient("normal", 2, rows, cols), gradient("mean", 2, rows, cols)
    m = M.clone()
    O = run(dtype, G, momentum=m, beta=0.75, nesterov=nesterov)
    want = 0.75 * M.double() + G.double()
    assert ((m.double() - want).abs() <= 2.0 ** -24 * 1.01 * want.abs()).all()              # one fused multiply-add
    U = G + 0.75 * m if nesterov else m
    check(dtype, O, U)


def test_matrices_do_not_touch_each_other():
    G = gradient("normal", 5, 150, 170)
    clean = run("bf16", G)
    G[1, 3, 4], G[3, 0, 0] = float("nan"), float("inf")
    G[2] = 0.0
    O = run("bf16", G)
    assert torch.equal(O[0], clean[0]) and torch.equal(O[4], clean[4])
    assert torch.isnan(O[1]).all() and torch.isnan(O[3]).all() and not O[2].any()
    for alone in (0, 4):
        assert torch.equal(run("bf16", G[alone:alone + 1].contiguous())[0], clean[alone])


def test_an_earlier_error_leaves_the_outputs_alone():
    G = gradient("normal", 1, 150, 170)
    m = torch.ones_like(G)
    status = torch.tensor([sbp.SBP_ERR_BAD_INDICES], dtype=torch.int32, device="cuda")
    O = run("bf16", G, momentum=m, status=status)
    assert torch.isnan(O).all() and (m == 1).all() and status.item() == sbp.SBP_ERR_BAD_INDICES


def test_captured_and_replayed():
    G = gradient("normal", 2, 256, 384)
    want = run("bf16", G)
    nbytes = sbp.sbp_orthogonalize_workspace_bytes(1, 2, 256, 384)
    ws, O = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.empty_like(want)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        sbp.sbp_orthogonalize(1, G, None, 0.0, 2, 256, 384, 5, 1e-7, 1.0, O, 0, ws, nbytes)
    for _ in range(2):
        O.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want)


@pytest.mark.parametrize("count,rows,cols", [(3, 640, 512), (20, 100, 700)])
def test_calls_at_once_on_three_streams(count, rows, cols):
    G = [gradient(how, count, rows, cols) for how in ("normal", "low", "mean")]
    want = [run("bf16", g) for g in G]
    nbytes = sbp.sbp_orthogonalize_workspace_bytes(1, count, rows, cols)
    ws = [torch.empty(nbytes, dtype=torch.uint8, device="cuda") for _ in G]
    O = [torch.full_like(w, float("nan")) for w in want]
    streams = [torch.cuda.Stream() for _ in G]
    torch.cuda.synchronize()
    for _ in range(4):
        for g, w, o, s in zip(G, ws, O, streams):
            with torch.cuda.stream(s):
                sbp.sbp_orthogonalize(1, g, None, 0.0, count, rows, cols, 5, 1e-7, 1.0, o, 0, w, nbytes)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(O, want))
