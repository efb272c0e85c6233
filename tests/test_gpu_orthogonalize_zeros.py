"""Matrices of zeros give zeros whatever eps above 0 is; with eps = 0 there is no direction, and the result is NaN."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,code", [(torch.bfloat16, 1), (torch.float32, 0)])
@pytest.mark.parametrize("rows,cols", [(40, 50), (150, 170), (100, 600)])
@pytest.mark.parametrize("eps", [1e-7, 1e-44, 1e-80, 1e-300, 5e-324, 1e300, 0.0])
def test_zeros(dtype, code, rows, cols, eps):
    G = torch.zeros((3, rows, cols), device="cuda")
    G[1] = torch.randn((rows, cols), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    O = torch.full(G.shape, float("nan"), dtype=dtype, device="cuda")
    nbytes = sbp.sbp_orthogonalize_workspace_bytes(code, 3, rows, cols)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    sbp.sbp_orthogonalize(code, G, None, 0.0, 3, rows, cols, 5, eps, 1.0, O, 0, ws, nbytes)
    torch.cuda.synchronize()
    if eps == 0.0:
        assert torch.isnan(O[0]).all() and torch.isnan(O[2]).all()
    else:
        assert not O[0].any() and not O[2].any()
    assert torch.isfinite(O[1]).all()
    if eps == 1e300:
        assert not O[1].any()                          # 1e-298 and below
