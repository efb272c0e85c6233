"""The bounds of norm_bounds.py hold for plain fp32 arithmetic, and a kept row that is left out, or a lost share of the rows, breaks them."""
import pytest
import torch

import norm_bounds


def made(K, C, kind, post, bias, group, dtype):
    g = torch.Generator().manual_seed(K + C)
    n = lambda *s, k=1.0, m=0.0, t=dtype: (torch.randn(s, generator=g) * k + m).to(t).double()
    f = torch.float32
    s = dict(R=n(K, C, k=2.0, m=0.3), Yk=n(K, C, m=0.3), dZ=n(K, C), pre_w=n(C, k=0.2, m=1.0, t=f), post_w=n(C, k=0.2, m=1.0, t=f) if post else None,
             post_b=n(C, t=f) if post and bias else None, gate=n(-(-2 * K // group), C, k=0.3, m=0.5) if group else None, group=max(group, 1))
    return s, torch.arange(0, 2 * K, 2), n(K, C)


def fp32(s, kind, rows, dR):
    """The same gradients in fp32, one operation after another."""
    t = {k: v.float() if torch.is_tensor(v) else v for k, v in s.items()}
    def normalise(x):
        d = x - x.mean(1, keepdim=True) if kind == 0 else x
        r = torch.rsqrt(d.square().mean(1, keepdim=True) + norm_bounds.EPS)
        return d * r, r
    n, r = normalise(t["R"])
    q = t["dZ"] * t["pre_w"]
    G = dR.float() + r * (q - (q.mean(1, keepdim=True) if kind == 0 else 0) - n * (q * n).mean(1, keepdim=True))
    out = dict(dpre_w=(t["dZ"] * n).sum(0), dpre_b=t["dZ"].sum(0))
    y = normalise(t["Yk"])[0] if t["post_w"] is not None else t["Yk"]
    u = y * t["post_w"] + (t["post_b"] if t["post_b"] is not None else 0) if t["post_w"] is not None else y
    gate = t["gate"][rows // t["group"]] if t["gate"] is not None else torch.ones_like(G)
    if t["gate"] is not None:
        out["dgate"] = torch.zeros_like(t["gate"]).index_add_(0, rows // t["group"], G * u)
    if t["post_w"] is not None:
        out["dpost_w"], out["dpost_b"] = (G * gate * y).sum(0), (G * gate).sum(0)
    return out


def without(s, rows, dR, gone):
    keep = torch.ones(rows.numel(), dtype=torch.bool)
    keep[gone] = False
    return dict(s, **{n: s[n][keep] for n in ("R", "Yk", "dZ")}), rows[keep], dR[keep]


@pytest.mark.parametrize("K,C,dtype", [(30000, 64, torch.bfloat16), (20000, 128, torch.float32), (7500, 256, torch.bfloat16), (1400, 768, torch.bfloat16),
                                       (700, 2048, torch.float32)])
@pytest.mark.parametrize("kind,post,bias,group", [(0, True, True, 7), (1, True, False, 1), (0, False, True, 0), (0, True, True, 10 ** 6)])
def test_fp32_holds_and_a_missing_row_does_not(K, C, dtype, kind, post, bias, group):
    s, rows, dR = made(K, C, kind, post, bias, group, dtype)
    want = norm_bounds.backward(s, kind, rows, dR)
    norm_bounds.check(fp32(s, kind, rows, dR), want)
    for gone in (slice(K // 2, K // 2 + 1), slice(K - 1, K), slice(K // 10, K // 9)):
        less, some, dR_some = without(s, rows, dR, gone)
        got = fp32(less, kind, some, dR_some)
        for name in got:
            with pytest.raises(AssertionError):
                norm_bounds.check({name: got[name]}, want)
