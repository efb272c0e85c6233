"""Results with both fp16 numbers of every operand lose nothing against fp32 arithmetic: their distance from the iteration in 64 bits is
at most one and a half times that of the same iteration in fp32 (products and sums rounded to nearest), and 2^-21 of the norm - eight
half steps of fp32, where the fp32 iteration happens to be nearer than its own roundings."""
import pytest
import torch

import test_gpu_orthogonalize as base

pytestmark = pytest.mark.gpu


def fp32_iteration(U, steps, eps=1e-7):
    a, b, c = base.NS
    tall = U.shape[1] > U.shape[2]
    X = U / (U.square().sum((1, 2), keepdim=True).sqrt() + eps)
    X = X.mT.contiguous() if tall else X
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X.mT if tall else X


@pytest.mark.parametrize("count,rows,cols", [(4, 64, 64), (4, 100, 100), (4, 128, 128), (4, 128, 256), (4, 100, 257), (4, 60, 500), (2, 128, 1000),
                                             (4, 2000, 128), (4, 30, 2048), (4, 129, 200), (2, 300, 300), (3, 533, 1926), (3, 1926, 533), (2, 256, 4096),
                                             (2, 1024, 1024), (1, 4096, 1024), (1, 131, 6000), (2, 700, 128)])
@pytest.mark.parametrize("how", ["normal", "low", "mean", "rows"])
@pytest.mark.parametrize("steps", [5, 8])
def test_no_further_from_64_bits_than_fp32(count, rows, cols, how, steps):
    allowed = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        G = base.gradient(how, count, rows, cols)
        plain = fp32_iteration(G, steps)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = allowed
    want = base.iterate(G, steps, 1e-7)
    off = lambda x: ((x.double() - want).square().sum((1, 2)).sqrt() / want.square().sum((1, 2)).sqrt()).max().item()
    got, limit = off(base.run("f32", G, steps=steps)), 1.5 * off(plain) + 2.0 ** -21
    assert got <= limit, (got, limit)
