"""Cache rows of list entries that lie outside the tensor: cleared by the forward call, so that what reads the caches meets numbers."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu


def inner_rows(M, before, behind, how):
    """Rows of the tensor in the list (a list has at most M entries)."""
    return {"some": list(range(0, M, 3)), "none": [], "all": list(range(max(0, M - before - behind)))}[how]


CASES = [(M, before, behind, how) for M in (1, 5, 37, 20000) for before, behind in ((0, 0), (1, 0), (3, 0), (0, 1), (0, 2), (40, 35))
         for how in ("some", "none", "all") if 0 < len(inner_rows(M, before, behind, how)) + before + behind <= M]


@pytest.mark.parametrize("dtype,code,C", [(torch.bfloat16, 1, 8), (torch.bfloat16, 1, 128), (torch.bfloat16, 1, 768), (torch.bfloat16, 1, 4104),
                                          (torch.float32, 0, 200), (torch.float32, 0, 516)])
@pytest.mark.parametrize("M,before,behind,how", CASES)
@pytest.mark.parametrize("counted", [False, True])
def test_rows_of_entries_outside_the_tensor_are_cleared(dtype, code, C, M, before, behind, how, counted):
    g = torch.Generator(device="cuda").manual_seed(M + C)
    n = lambda *s: torch.randn(s, device="cuda", generator=g)
    inner = inner_rows(M, before, behind, how)
    ids = [-2 ** 31 + i for i in range(before)] + inner + [M + i for i in range(behind)]
    if behind > 1:
        ids[-1] = 2 ** 31 - 1
    keep, cap = len(ids), min(M, len(ids) + 2) if counted else len(ids)
    rows = torch.tensor(ids + [0] * (cap - keep), dtype=torch.int64, device="cuda").int()
    count = torch.tensor([keep], dtype=torch.int32, device="cuda") if counted else None
    H, Y, w = n(M, C).to(dtype), n(M, C).to(dtype), n(C)
    R, Z = torch.empty_like(H), torch.empty_like(H)
    caches = [torch.full((cap, C), float("nan"), dtype=dtype, device="cuda") for _ in range(3)]
    sbp.sbp_block_norm_forward(code, 0, H, Y, w, None, None, 1, 0.9, w, None, 1e-6, M, C, R, Z, rows, count, cap, *caches)
    torch.cuda.synchronize()
    at = slice(before, before + len(inner))
    for cache, full in zip(caches, (Y, R, Z)):
        assert torch.equal(cache[at], full[torch.tensor(inner, dtype=torch.int64, device="cuda")])
        cache[at] = 0
        assert not torch.isnan(cache).any() and not cache.any()
