"""Performance cases of the operators around the SBP layers of a training step.

``norm_fwd`` / ``norm_bwd``  norms before and after a block with its gate and residual scale:
        u = norm(Y) w_post + b_post,  R = s H + gate u,  Z = norm(R) w_pre + b_pre
    with the kept rows of Y, R and Z cached, and the gradients on those rows.
``embed_fwd`` / ``embed_bwd``  rows of a table by id, scaled, plus an addend; the table's gradient from the kept rows.
``ortho``  Newton-Schulz orthogonalisation of (momentum-averaged) weight gradients.

With ``own`` false the operators are computed in elementary torch operations in 32 bits; with ``own`` true through the
library.  Both take the same state, and return new values of the same outputs.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6
_NS = (3.4445, -4.7750, 2.0315)      # the quintic's coefficients


# ---- the listed cases ------------------------------------------------------------------------------------------------
def _norm(kind, name, dtype, norm, B, N, C, ratio, post, gate, bias):
    c = dict(kind=kind, dtype=dtype, norm=norm, B=B, N=N, C=C, ratio=ratio, post=post, gate=gate, bias=bias)
    return dict(c, name=name) if name else c


def _ortho(name, dtype, count, rows, cols, nesterov):
    c = dict(kind="ortho", dtype=dtype, count=count, rows=rows, cols=cols, nesterov=nesterov)
    return dict(c, name=name) if name else c


def _embed(kind, name, dtype, V, B, N, C, ids, ratio, add):
    c = dict(kind=kind, dtype=dtype, V=V, B=B, N=N, C=C, ids=ids, ratio=ratio, add=add)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one image of 197 tokens through a ViT-B/16 block's norm: the smallest call, bound by latency
        _norm("norm_fwd", "norm_fwd_one_image", "bf16", "layer", 1, 197, 768, 0.5, False, "channel", True),
        # the benchmark's batch: norm after and before the block, a gate for each sample
        _norm("norm_fwd", "norm_fwd_vit_b128", "bf16", "layer", 128, 196, 768, 0.5, True, "sample", True),
        # wide RMS-normalised rows of a language model, no rows dropped
        _norm("norm_fwd", "norm_fwd_rms_4096", "bf16", "rms", 4, 2047, 4096, 1.0, True, "none", False),
        # the gradients of the first two
        _norm("norm_bwd", "norm_bwd_one_image", "bf16", "layer", 1, 197, 768, 0.5, False, "channel", True),
        _norm("norm_bwd", "norm_bwd_vit_b128", "bf16", "layer", 128, 196, 768, 0.5, True, "sample", True),
        # ConvNeXt-B stage 1 in fp32: few channels, many positions, a learned scale for each channel (layer scale)
        _norm("norm_bwd", "norm_bwd_convnext_s1_f32", "f32", "layer", 64, 3136, 128, 0.5, True, "channel", True),
        # the projection weights of twelve ViT-B/16 blocks in one call
        _ortho("ortho_vit_proj_x12", "bf16", 12, 768, 768, True),
        # one small odd-sized matrix
        _ortho("ortho_100x257", "bf16", 1, 100, 257, False),
        # tall matrices (stage-4 ConvNeXt MLP), the update kept in fp32
        _ortho("ortho_4096x1024_f32", "f32", 2, 4096, 1024, True),
        # tokens of a language model, looked up and scaled
        _embed("embed_fwd", "embed_fwd_50257", "bf16", 50257, 16, 1024, 768, "zipf", 1.0, False),
        # a ViT's position table: every position once a sample, half of the rows kept, added into few rows
        _embed("embed_bwd", "embed_bwd_positions", "bf16", 196, 128, 196, 768, "position", 0.5, False),
        # a language model's table: most ids rare, a few very frequent
        _embed("embed_bwd", "embed_bwd_50257", "bf16", 50257, 16, 1024, 768, "zipf", 0.75, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_fwd", "norm_bwd", "ortho", "embed_fwd", "embed_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    ratio = rng.choice([0.25, 0.5, 0.75, 1.0])
    if kind in ("norm_fwd", "norm_bwd"):
        C = 8 * _log(rng, 8, 640)
        M = _log(rng, 16, max(17, min(40000, (24 << 20) // (C * (2 if dtype == "f32" else 1)))))
        N = min(M, _log(rng, 1, 2048))
        return _norm(kind, None, dtype, rng.choice(["layer", "rms"]), max(1, M // N), N, C, ratio, rng.random() < 0.6,
                     rng.choice(["none", "sample", "channel"]), rng.random() < 0.6)
    if kind == "ortho":
        rows, cols = _log(rng, 16, 2048), _log(rng, 16, 2048)
        work = min(rows, cols) ** 2 * max(rows, cols)
        return _ortho(None, dtype, rng.randint(1, max(1, min(12, 2 * 1024 * 1024 * 4096 // work))), rows, cols, rng.random() < 0.5)
    C = 8 * _log(rng, 8, 128)
    T = _log(rng, 16, 16384)
    N = min(T, _log(rng, 1, 1024))
    V = _log(rng, 8, 40000)
    return _embed(kind, None, dtype, V, max(1, T // N), N, C, rng.choice(["zipf", "uniform", "position"]), ratio, rng.random() < 0.5)


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _keep(g, B, N, ratio):
    """Ascending row ids of a uniformly random subset of every sample's rows, as the sampler draws them."""
    K = min(N, max(1, int(ratio * N + 0.5)))
    order = torch.rand((B, N), device="cuda", generator=g).argsort(1)[:, :K].sort(1).values
    return (order + torch.arange(B, device="cuda")[:, None] * N).reshape(-1).to(torch.int32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}

    def normal(*shape, scale=1.0, mean=0.0, dtype=torch.float32):
        return torch.randn(shape, device="cuda", generator=g).mul_(scale).add_(mean).to(dtype)

    if kind == "ortho":
        n, r, c = case["count"], case["rows"], case["cols"]
        k = min(r, c, 8)
        # a weight gradient: a few strong directions over noise
        G = normal(n, r, c, scale=1e-3)
        G += torch.bmm(normal(n, r, k, scale=1e-3), normal(n, k, c))
        s["G"], s["momentum"] = G, normal(n, r, c, scale=1e-2)
        return s
    dt = _DT[case["dtype"]]
    B, N, C = case["B"], case["N"], case["C"]
    M = B * N
    s["rows"] = _keep(g, B, N, case["ratio"])
    K = s["rows"].numel()
    if kind in ("norm_fwd", "norm_bwd"):
        groups = {"none": 0, "sample": B, "channel": 1}[case["gate"]]
        s["gate"] = normal(groups, C, scale=0.3, mean=0.5, dtype=dt) if groups else None
        s["gate_group"] = {"none": 1, "sample": N, "channel": M}[case["gate"]]
        for w in ("post", "pre"):
            has = w == "pre" or case["post"]
            s[w + "_w"] = normal(C, scale=0.2, mean=1.0) if has else None
            s[w + "_b"] = normal(C, scale=0.1) if has and case["bias"] else None
        s["scale"] = 1.0 if case["gate"] == "channel" else 0.9
        if kind == "norm_fwd":
            s["H"], s["Y"] = normal(M, C, scale=2.0, mean=0.3, dtype=dt), normal(M, C, dtype=dt)
        else:
            s["dR"], s["dZ"] = normal(M, C, scale=1e-2, dtype=dt), normal(K, C, scale=1e-2, dtype=dt)
            s["R"], s["Y"] = normal(K, C, scale=2.0, mean=0.3, dtype=dt), normal(K, C, dtype=dt)
        return s
    V = case["V"]
    if case["ids"] == "position":
        ids = torch.arange(N, device="cuda").repeat(B) % V
    elif case["ids"] == "uniform":
        ids = torch.randint(0, V, (M,), device="cuda", generator=g)
    else:                               # frequencies that fall with the rank, ranks scattered over the table
        u = torch.rand(M, device="cuda", generator=g, dtype=torch.float64)
        rank = torch.exp(u * math.log(V)).long().clamp_(1, V) - 1
        ids = torch.randperm(V, device="cuda", generator=g)[rank]
    ids[torch.rand(M, device="cuda", generator=g) < 0.01] = -1          # padding
    s["ids"] = ids.to(torch.int32)
    s["scale"] = math.sqrt(C)
    if kind == "embed_fwd":
        s["table"] = normal(V, C, scale=0.02, dtype=dt)
        s["add"] = normal(M, C, dtype=dt) if case["add"] else None
    else:
        s["dOut"] = normal(M, C, scale=1e-2, dtype=dt)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------------
def _statistics(x, norm):
    mean = x.mean(-1, keepdim=True) if norm == "layer" else torch.zeros_like(x[:, :1])
    centred = x - mean
    return centred, torch.rsqrt(centred.square().mean(-1, keepdim=True) + _EPS)


def _affine(x, w, b):
    x = x * w
    return x if b is None else x + b


def _gate_of(s, rows, M):
    return None if s["gate"] is None else s["gate"].float()[torch.div(rows, s["gate_group"], rounding_mode="floor")]


def _plain_norm_fwd(s):
    case, rows, dt = s["case"], s["rows"].long(), s["H"].dtype
    u = s["Y"].float()
    if s["post_w"] is not None:
        c, r = _statistics(u, case["norm"])
        u = _affine(c * r, s["post_w"], s["post_b"])
    if s["gate"] is not None:
        u = (u.view(s["gate"].shape[0], -1, u.shape[1]) * s["gate"].float()[:, None, :]).view(u.shape)
    R = s["scale"] * s["H"].float() + u
    c, r = _statistics(R, case["norm"])
    Z = _affine(c * r, s["pre_w"], s["pre_b"]).to(dt)
    R = R.to(dt)
    return {"R": R, "Z": Z, "R_keep": R[rows], "Y_keep": s["Y"][rows], "Z_keep": Z[rows]}


def _norm_grad(c, r, g, norm):
    """Gradient of the normalised rows c r with respect to the rows, g that with respect to the normalised rows."""
    xhat = c * r
    inner = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if norm == "layer":
        inner = inner - g.mean(-1, keepdim=True)
    return inner * r


def _plain_norm_bwd(s):
    case, rows, dt = s["case"], s["rows"].long(), s["dR"].dtype
    dR, dZ = s["dR"].to(torch.float32, copy=True), s["dZ"].float()       # (the gradient is written over below)
    c, r = _statistics(s["R"].float(), case["norm"])
    G = dR[rows] + _norm_grad(c, r, dZ * s["pre_w"], case["norm"])
    out = {"dpre_w": (dZ * (c * r)).sum(0), "dpre_b": dZ.sum(0) if s["pre_b"] is not None else None}
    dR[rows] = G
    out["dH"] = (s["scale"] * dR).to(dt)
    u = s["Y"].float()
    if s["post_w"] is not None:
        c, r = _statistics(u, case["norm"])
        u = _affine(c * r, s["post_w"], s["post_b"])
    if s["gate"] is not None:
        groups = torch.div(rows, s["gate_group"], rounding_mode="floor")
        out["dgate"] = (G * u).view(s["gate"].shape[0], -1, u.shape[1]).sum(1)
        G = G * s["gate"].float()[groups]
    if s["post_w"] is not None:
        out["dpost_w"], out["dpost_b"] = (G * (c * r)).sum(0), G.sum(0) if s["post_b"] is not None else None
        G = _norm_grad(c, r, G * s["post_w"], case["norm"])
    out["dY"] = G.to(dt)
    return out


def _plain_embed_fwd(s):
    ids = s["ids"].long()
    out = s["scale"] * s["table"][ids.clamp_min(0)].float()
    out = torch.where(ids[:, None] >= 0, out, torch.zeros((), device="cuda"))
    if s["add"] is not None:
        out = out + s["add"].float()
    return out.to(s["table"].dtype)


def _plain_embed_bwd(s):
    rows = s["rows"].long()
    ids = s["ids"].long()[rows]
    V = s["case"]["V"]
    dTable = torch.zeros((V + 1, s["dOut"].shape[1]), device="cuda")        # the last row takes the padding
    dTable.index_add_(0, torch.where(ids >= 0, ids, V), s["dOut"][rows].float() * s["scale"])
    return dTable[:V]


def _plain_ortho(s):
    case = s["case"]
    s["momentum"].mul_(0.95).add_(s["G"])
    X = s["G"] + 0.95 * s["momentum"] if case["nesterov"] else s["momentum"]
    X = X / (torch.sqrt(X.square().sum((1, 2), keepdim=True)) + 1e-7)
    tall = case["rows"] > case["cols"]
    if tall:
        X = X.mT
    a, b, c = _NS
    for _ in range(5):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    X = (X.mT if tall else X) * max(1.0, case["rows"] / case["cols"]) ** 0.5
    return {"O": X.to(_DT[case["dtype"]]).contiguous(), "momentum": s["momentum"]}


# ---- through the library ---------------------------------------------------------------------------------------------
def _own_buffers(s):
    """Outputs and workspace, made at the first pass and kept, as a training program keeps them."""
    import paper_2210_00129_b200 as sbp
    case, o = s["case"], {}

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    o["dt"] = sbp.SBP_BF16 if case["dtype"] == "bf16" else sbp.SBP_F32
    dt = _DT[case["dtype"]]
    o["ws"], o["nbytes"] = None, 0
    if case["kind"] == "ortho":
        o["O"] = empty(case["count"], case["rows"], case["cols"], dtype=dt)
        o["nbytes"] = sbp.sbp_orthogonalize_workspace_bytes(o["dt"], case["count"], case["rows"], case["cols"])
    else:
        M, K, C = case["B"] * case["N"], s["rows"].numel(), case["C"]
        if case["kind"] == "norm_fwd":
            o["norm"] = sbp.SBP_NORM_LAYER if case["norm"] == "layer" else sbp.SBP_NORM_RMS
            o["out"] = {n: empty(M if n in "RZ" else K, C, dtype=dt) for n in ("R", "Z", "R_keep", "Y_keep", "Z_keep")}
        elif case["kind"] == "norm_bwd":
            o["norm"] = sbp.SBP_NORM_LAYER if case["norm"] == "layer" else sbp.SBP_NORM_RMS
            out = o["out"] = {"dH": empty(M, C, dtype=dt), "dY": empty(K, C, dtype=dt)}
            for w in ("post_w", "post_b", "pre_w", "pre_b", "gate"):
                out["d" + w] = empty(*s[w].shape) if s[w] is not None else None
            o["nbytes"] = sbp.sbp_block_norm_backward_workspace_bytes(o["dt"], M, K, C)
        elif case["kind"] == "embed_fwd":
            o["out"] = empty(M, C, dtype=dt)
        else:
            o["out"] = empty(case["V"], C)
            o["nbytes"] = sbp.sbp_embedding_backward_workspace_bytes(o["dt"], K, case["V"], C)
    if o["nbytes"]:
        o["ws"] = torch.empty(o["nbytes"], dtype=torch.uint8, device="cuda")
    s["own"] = o
    return o


def _run_own(s):
    import paper_2210_00129_b200 as sbp
    o = s.get("own") or _own_buffers(s)
    case = s["case"]
    kind = case["kind"]
    if kind == "ortho":
        scale = max(1.0, case["rows"] / case["cols"]) ** 0.5
        sbp.sbp_orthogonalize(o["dt"], s["G"], s["momentum"], 0.95, case["count"], case["rows"], case["cols"], 5, 1e-7, scale,
                              o["O"], sbp.SBP_FLAG_NESTEROV if case["nesterov"] else 0, o["ws"], o["nbytes"])
        return {"O": o["O"], "momentum": s["momentum"]}
    M, K, C, out = case["B"] * case["N"], s["rows"].numel(), case["C"], o["out"]
    if kind == "norm_fwd":
        sbp.sbp_block_norm_forward(o["dt"], o["norm"], s["H"], s["Y"], s["post_w"], s["post_b"], s["gate"], s["gate_group"],
                                   s["scale"], s["pre_w"], s["pre_b"], _EPS, M, C, out["R"], out["Z"], s["rows"], None, K,
                                   out["Y_keep"], out["R_keep"], out["Z_keep"])
    elif kind == "norm_bwd":
        sbp.sbp_block_norm_backward(o["dt"], o["norm"], s["dR"], s["dZ"], s["R"], s["Y"], s["post_w"], s["post_b"], s["gate"],
                                    s["gate_group"], s["scale"], s["pre_w"], _EPS, s["rows"], None, M, K, C, out["dH"],
                                    out["dY"], out["dpost_w"], out["dpost_b"], out["dgate"], out["dpre_w"], out["dpre_b"], 0,
                                    o["ws"], o["nbytes"])
    elif kind == "embed_fwd":
        sbp.sbp_embedding_forward(o["dt"], s["table"], case["V"], C, s["ids"], M, s["scale"], s["add"], out)
    else:
        sbp.sbp_embedding_backward(o["dt"], s["dOut"], s["ids"], s["rows"], None, M, K, case["V"], C, s["scale"], out, 0,
                                   o["ws"], o["nbytes"])
    return out


def run(state):
    if own:
        return _run_own(state)
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "embed_fwd": _plain_embed_fwd,
            "embed_bwd": _plain_embed_bwd, "ortho": _plain_ortho}[state["case"]["kind"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    size = 2 if case["dtype"] == "bf16" else 4
    if kind == "ortho":
        m, n = sorted((case["rows"], case["cols"]))
        # gradient and momentum in, momentum and update out; the products of symmetric results made once
        return {"bytes": case["count"] * m * n * (12 + size), "flops": case["count"] * 5 * (m * m * n + m ** 3 + 2 * m * m * n)}
    B, N, C = case["B"], case["N"], case["C"]
    M, K = B * N, B * min(N, max(1, int(case["ratio"] * N + 0.5)))
    if kind == "norm_fwd":
        return {"bytes": (4 * M + 3 * K) * C * size, "flops": 20 * M * C}
    if kind == "norm_bwd":
        return {"bytes": (2 * M + 4 * K) * C * size, "flops": 40 * K * C}
    V = case["V"]
    if kind == "embed_fwd":
        return {"bytes": (M * (2 if case["add"] else 1) + min(M, V)) * C * size + 4 * M, "flops": 2 * M * C}
    return {"bytes": K * C * size + 8 * K + 4 * V * C, "flops": 2 * K * C}


# ---- in 64 bits ------------------------------------------------------------------------------------------------------
def _norm64(x, w, b, kind):
    """The definition, for autograd to differentiate."""
    n = x.shape[1]
    if kind == "layer":
        x = x - x.sum(1, keepdim=True) / n
    y = x / ((x * x).sum(1, keepdim=True) / n + _EPS) ** 0.5 * w.double()
    return y if b is None else y + b.double()


def _block64(H, Y, s, gate, weights, kind, rows):
    u = Y
    if s["post_w"] is not None:
        u = _norm64(Y, weights["post_w"], weights["post_b"], kind)
    if gate is not None:
        u = u * gate[rows // s["gate_group"]]
    R = s["scale"] * H + u
    return R


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "ortho":
        mom = s["momentum"].double() * 0.95 + s["G"].double()
        X = s["G"].double() + 0.95 * mom if case["nesterov"] else mom
        X = X / (X.reshape(X.shape[0], -1).norm(dim=1)[:, None, None] + 1e-7)
        # on the smaller side's Gram matrix: X p(S) with S = X^T X where that is smaller, else p(S) X with S = X X^T
        a, b, c = _NS
        for _ in range(5):
            if X.shape[1] > X.shape[2]:
                S = torch.einsum("kij,kil->kjl", X, X)
                X = a * X + X @ S * b + X @ S @ S * c
            else:
                S = torch.einsum("kij,klj->kil", X, X)
                X = a * X + S @ X * b + S @ (S @ X) * c
        return {"O": X * max(1.0, case["rows"] / case["cols"]) ** 0.5, "momentum": mom}
    rows = s["rows"].long()
    if kind == "norm_fwd":
        H, Y = s["H"].double(), s["Y"].double()
        gate = None if s["gate"] is None else s["gate"].double()
        R = _block64(H, Y, s, gate, s, case["norm"], torch.arange(H.shape[0], device="cuda"))
        Z = _norm64(R, s["pre_w"], s["pre_b"], case["norm"])
        return {"R": R, "Z": Z, "R_keep": R[rows], "Y_keep": Y[rows], "Z_keep": Z[rows]}
    if kind == "norm_bwd":
        leaf = {n: s[n].double().requires_grad_() if s[n] is not None else None
                for n in ("post_w", "post_b", "pre_w", "pre_b", "gate", "R", "Y")}
        Z = _norm64(leaf["R"], leaf["pre_w"], leaf["pre_b"], case["norm"])
        wanted = [n for n in ("R", "pre_w", "pre_b") if leaf[n] is not None]
        grads = dict(zip(wanted, torch.autograd.grad(Z, [leaf[n] for n in wanted], s["dZ"].double())))
        G = grads.pop("R") + s["dR"].double()[rows]
        dH = s["dR"].double()
        dH[rows] = G
        R = _block64(torch.zeros_like(leaf["Y"]), leaf["Y"], s, leaf["gate"], leaf, case["norm"], rows)
        wanted = [n for n in ("post_w", "post_b", "gate", "Y") if leaf[n] is not None]
        grads |= dict(zip(wanted, torch.autograd.grad(R, [leaf[n] for n in wanted], G)))
        return {"dH": s["scale"] * dH} | {"d" + n: g for n, g in grads.items()}
    ids = s["ids"].long()
    if kind == "embed_fwd":
        known = (ids >= 0).nonzero()[:, 0]
        out = torch.zeros((ids.numel(), case["C"]), dtype=torch.float64, device="cuda") if s["add"] is None else s["add"].double()
        out[known] += s["table"].double()[ids[known]] * s["scale"]
        return out
    rows = rows[ids[rows] >= 0]
    order = ids[rows].sort(stable=True)
    sums = torch.cumsum(s["dOut"].double()[rows[order.indices]] * s["scale"], 0)      # differences of running sums
    out = torch.zeros((case["V"], case["C"]), dtype=torch.float64, device="cuda")
    value, count = torch.unique_consecutive(order.values, return_counts=True)
    end = torch.cumsum(count, 0) - 1
    at_end = sums[end]
    out[value] = at_end - torch.cat([torch.zeros_like(at_end[:1]), at_end[:-1]])
    return out
