"""Tensors of more than 2^31 elements: rows far into them come out as the same rows do in a small call, or as the formula gives them."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(torch.cuda.is_available() and torch.cuda.get_device_properties(0).total_memory < 10 ** 11,
                                                  reason="needs 60 GB of device memory")]

C = 8192
M = 2 ** 31 // C + 300                                 # rows
BF16 = sbp.SBP_BF16


def rows_of(M, seed):
    """Random rows; one block of them over and over, which takes no time to draw."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    few = torch.randn((1000, C), device="cuda", generator=g).bfloat16()
    out = torch.empty((M, C), dtype=torch.bfloat16, device="cuda")
    for i in range(0, M, 1000):
        out[i:i + 1000] = few[:min(1000, M - i)]
    return out


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [900, 5000])
def test_embedding(n):
    table = rows_of(M, 1)
    g = torch.Generator(device="cuda").manual_seed(n)
    ids = torch.randint(M - 20000, M, (n,), device="cuda", generator=g).unique().int()
    ids[-1], n = M - 1, len(ids)
    ids = ids[torch.rand(n, device="cuda", generator=g).argsort()].contiguous()
    out = torch.empty((n, C), dtype=torch.bfloat16, device="cuda")
    sbp.sbp_embedding_forward(BF16, table, M, C, ids, n, 2.0, None, out)
    assert torch.equal(out, table[ids.long()] * 2)
    del table
    nbytes = sbp.sbp_embedding_backward_workspace_bytes(BF16, n, M, C)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    grad = torch.full((M, C), float("nan"), device="cuda")
    sbp.sbp_embedding_backward(BF16, out, ids, None, None, n, n, M, C, 0.5, grad, 0, ws, nbytes)
    assert torch.equal(grad[ids.long()], out.float() * 0.5)
    grad[ids.long()] = 0
    assert not any(part.any() for part in grad.split(20000))


def test_embedding_gradient_of_many_rows():
    V = 5
    grad = rows_of(M, 2)
    ids = (torch.arange(M, device="cuda") * 7 % V).int()
    nbytes = sbp.sbp_embedding_backward_workspace_bytes(BF16, M, V, C)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    table = torch.full((V, C), float("nan"), device="cuda")
    sbp.sbp_embedding_backward(BF16, grad, ids, None, None, M, M, V, C, 1.0, table, 0, ws, nbytes)
    want, size = torch.zeros((V, C), dtype=torch.float64, device="cuda"), torch.zeros((V, C), dtype=torch.float64, device="cuda")
    for i in range(0, M, 10000):
        x = grad[i:i + 10000].double()
        want.index_add_(0, ids[i:i + 10000].long(), x)
        size.index_add_(0, ids[i:i + 10000].long(), x.abs())
    # 8192 columns are 32 strips of a warp, so the list is cut into 16 * 148 / 32 = 74 pieces: 3547 rows one after another in each,
    # then the pieces of an id; half a step an addition
    assert ((table.double() - want).abs() <= (3547 + 74 + 8) * 2.0 ** -24 * size).all()


def test_block_norm():
    H, Y, gate = rows_of(M, 3), rows_of(M, 4), rows_of(M, 5)
    g = torch.Generator(device="cuda").manual_seed(6)
    weights = [torch.rand(C, device="cuda", generator=g) + 0.5 for _ in range(4)]
    rows = torch.randint(0, M, (700,), device="cuda", generator=g).unique()
    rows[-1] = M - 1
    keep = len(rows)
    new = lambda n, dt=torch.bfloat16: torch.full((n, C), float("nan"), dtype=dt, device="cuda")

    def forward(H, Y, gate, rows, M):
        R, Z, caches = new(M), new(M), [new(len(rows)) for _ in range(3)]
        sbp.sbp_block_norm_forward(BF16, sbp.SBP_NORM_LAYER, H, Y, weights[0], weights[1], gate, 1, 0.9, weights[2], weights[3], 1e-6, M, C, R, Z,
                                   rows, None, len(rows), *caches)
        return R, Z, caches

    R, Z, caches = forward(H, Y, gate, rows.int(), M)
    every = torch.arange(keep, device="cuda").int()
    R2, Z2, caches2 = forward(H[rows], Y[rows], gate[rows], every, keep)
    assert torch.equal(R[rows], R2) and torch.equal(Z[rows], Z2)
    assert all(torch.equal(a, b) for a, b in zip(caches, caches2))
    assert not any(part.isnan().any() for part in R.split(20000)) and not any(part.isnan().any() for part in Z.split(20000))
    del H, R, Z, R2, Z2
    dZ = torch.randn((keep, C), device="cuda", generator=g).bfloat16()

    def backward(dR, gate, rows, M):
        dH, dY, dgate, sums = new(M), new(keep), new(M, torch.float32), [torch.full((C,), float("nan"), device="cuda") for _ in range(4)]
        nbytes = sbp.sbp_block_norm_backward_workspace_bytes(BF16, M, keep, C)
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        sbp.sbp_block_norm_backward(BF16, sbp.SBP_NORM_LAYER, dR, dZ, caches[1], caches[0], weights[0], weights[1], gate, 1, 0.9, weights[2], 1e-6,
                                    rows, None, M, keep, C, dH, dY, sums[0], sums[1], dgate, sums[2], sums[3], 0, ws, nbytes)
        return dH, dY, dgate, sums

    dH, dY, dgate, sums = backward(Y, gate, rows.int(), M)
    dH2, dY2, dgate2, sums2 = backward(Y[rows], gate[rows], every, keep)
    assert torch.equal(dH[rows], dH2) and torch.equal(dY, dY2) and torch.equal(dgate[rows], dgate2)
    assert all(torch.equal(a, b) for a, b in zip(sums, sums2))
    dgate[rows] = 0
    assert not any(part.any() for part in dgate.split(20000))
    Y[rows] = 0
    dH[rows] = 0
    for a, b in zip(dH.split(20000), Y.split(20000)):
        assert torch.equal(a, (b.float() * 0.9).bfloat16())


def test_orthogonalisation():
    count, side = 33, 4096                             # 33 * 4 planes of X: 2.2e9 numbers
    g = torch.Generator(device="cuda").manual_seed(7)
    G = torch.randn((1, side, side), device="cuda", generator=g).expand(count, -1, -1).contiguous()
    G[1:-1] *= 2.0 ** torch.arange(1, count - 1, device="cuda")[:, None, None]            # (the same direction: the same result)
    nbytes = sbp.sbp_orthogonalize_workspace_bytes(BF16, count, side, side)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    O = torch.full(G.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    sbp.sbp_orthogonalize(BF16, G, None, 0.0, count, side, side, 5, 0.0, 1.0, O, 0, ws, nbytes)
    assert not O[0].isnan().any()
    assert all(torch.equal(O[0], O[i]) for i in range(1, count))
    X = G[0].double() / G[0].double().norm()
    for _ in range(5):
        A = X @ X.mT
        X = 3.4445 * X + (-4.7750 * A + 2.0315 * (A @ A)) @ X
    assert ((O[0].double() - X).norm() <= 5e-3 * X.norm()).all()
