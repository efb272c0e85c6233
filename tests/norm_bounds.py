"""How far fp32 arithmetic may be from the gradients of the norms' weights and of the gate, column by column.

All in 64 bits, to first order in u = 2^-24 and rounded up by a tenth.  A row's sums have at most D = 40 additions one after
another (16 numbers of a thread, five exchanges, 16 warps).  With x a row, m its mean, d = x - m, s its deviation, n = d / s:
  m:  off by (D + 2) u mean|x| (the sum, 1 / C and the product);  e = that over s
  s:  the squares' sum relatively by (D + 4) u + 2 e (2 d dm summed: |d| s at most), its inverse root by half of that and 4 u (rsqrtf)
  n:  off by e + |n| (e + (D / 2 + 8) u)
A column's gradient is a sum over rows of terms; it may be off by the sum of the terms' own errors, and by (additions one after
another) u sum |terms|."""
import torch

U = 2.0 ** -24
D = 40.0
EPS = 1e-6


def normalised(x, kind):
    """n, its error, the inverse deviation and its relative error"""
    m = x.mean(1, keepdim=True) if kind == 0 else torch.zeros_like(x[:, :1])
    d = x - m
    s = (d.square().mean(1, keepdim=True) + EPS).sqrt()
    e = (D + 2) * U * x.abs().mean(1, keepdim=True) / s if kind == 0 else torch.zeros_like(s)
    n = d / s
    return n, e + n.abs() * (e + (D / 2 + 8) * U), 1 / s, e + (D / 2 + 6) * U


def additions(K, C):
    """One after another in a column's sum: a worker's rows (and as many gate rows again), a block's workers, the blocks' rows.  A block
    has eight workers or more up to 256 channels, two up to 768 (bf16 and fp32), one beyond; there are 148 where K is not smaller."""
    each = 8 if C <= 256 else 2 if C <= 768 else 1
    return 2 * -(-K // (148 * each)) + 48 + 24


def backward(s, kind, rows, dR_rows, with_z=True):
    """Gradients of the five weights and how far each may be off.  s: 64-bit tensors, the kept rows of R, Y and dZ, the weights;
    rows: the kept ones; dR_rows: their dR."""
    C = s["Yk"].shape[1]
    K = rows.numel()
    G, dG = dR_rows, torch.zeros_like(dR_rows)
    out = {}

    def total(name, terms, errors):
        out[name] = (terms.sum(0), 1.1 * (errors.sum(0) + additions(K, C) * U * terms.abs().sum(0)))

    if with_z:
        n, dn, r, dr = normalised(s["R"], kind)
        dZ = s["dZ"]
        total("dpre_w", dZ * n, dZ.abs() * dn + U * (dZ * n).abs())
        total("dpre_b", dZ, torch.zeros_like(dZ))
        q = dZ * s["pre_w"]
        mean = lambda x: x.mean(1, keepdim=True)
        mq = mean(q) if kind == 0 else torch.zeros_like(q[:, :1])
        dmq = (D + 3) * U * mean(q.abs()) if kind == 0 else torch.zeros_like(mq)
        mqn, dmqn = mean(q * n), mean(q.abs() * dn) + (D + 4) * U * mean((q * n).abs())
        parts = (q.abs() * (2 * U + dr) + mq.abs() * (3 * U + dr) + dmq + (n * mqn).abs() * (5 * U + dr) + dn * mqn.abs() + n.abs() * dmqn) * r
        G = G + r * (q - mq - n * mqn)
        dG = parts + 2 * U * G.abs()
    if s["post_w"] is not None:
        y, dy, _, _ = normalised(s["Yk"], kind)
    else:
        y, dy = s["Yk"], torch.zeros_like(s["Yk"])
    gates = torch.ones_like(G) if s["gate"] is None else s["gate"][rows // s["group"]]
    post_w = s["post_w"] if s["post_w"] is not None else torch.ones(C, dtype=torch.float64, device=G.device)
    post_b = s["post_b"] if s["post_b"] is not None else torch.zeros(C, dtype=torch.float64, device=G.device)
    dGy = dG * y.abs() + G.abs() * dy + U * (G * y).abs()
    if s["post_w"] is not None:
        total("dpost_w", G * y * gates, dGy * gates.abs() + 2 * U * (G * y * gates).abs())
        total("dpost_b", G * gates, dG * gates.abs() + 2 * U * (G * gates).abs())
    if s["gate"] is not None:
        each = rows // s["group"]
        put = lambda x: torch.zeros(s["gate"].shape, dtype=torch.float64, device=G.device).index_add_(0, each, x)
        size = (G * y * post_w).abs() + (G * post_b).abs()
        most = torch.bincount(each).max().item()       # rows of a gate row: no more are added up
        out["dgate"] = (put(G * y * post_w + G * post_b),
                        1.1 * put(dGy * post_w.abs() + dG * post_b.abs() + (4 + min(2 * most + 72, additions(K, C))) * U * size))
    return out


def check(got, bounds, add=0.0):
    """`got`: fp32 gradients by name; add: what was accumulated into."""
    for name, (want, off) in bounds.items():
        if got.get(name) is None:
            continue
        wrong = (got[name].double() - want - add).abs() - off - 2 * U * ((want + add).abs() + abs(add))
        assert not torch.isnan(got[name]).any(), name
        assert (wrong <= 0).all(), (name, wrong.max().item(), off.max().item(), want.abs().max().item())
