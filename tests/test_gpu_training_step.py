"""The operators together, as a training step uses them: embedding, norm, linear layer, norm after the block with its gate and the
residual stream, linear layer; then back through all of them on the kept rows, down to the table, and the updates of the weights.
The reference is the same network in 64 bits, differentiated by autograd, with the block's and the loss's gradients masked to
the kept rows (the residual stream's own gradient passes everywhere).

Tolerances: the library's relative Frobenius error of one operator (1e-5 fp32, 5e-3 bf16), once for each operator a value has come
through (eight on the way to the table's gradient)."""
import pytest
import torch

import paper_2210_00129_b200 as sbp

pytestmark = pytest.mark.gpu

DT = {"bf16": (sbp.SBP_BF16, torch.bfloat16, 5e-3), "f32": (sbp.SBP_F32, torch.float32, 1e-5)}
EPS = 1e-5


class Step:
    """Every buffer of the step, made once; forward() and backward() are the library's calls."""

    def __init__(self, dtype, B, N, C, hidden, V, kind, ratio=0.5):
        self.code, self.dt, self.tol = DT[dtype]
        self.B, self.N, self.C, self.hidden, self.V, self.kind = B, N, C, hidden, V, kind
        self.M = M = B * N
        g = torch.Generator(device="cuda").manual_seed(C + N)
        n = lambda *s, k=1.0, m=0.0: torch.randn(s, device="cuda", generator=g) * k + m
        self.p = dict(table=n(V, C, k=0.5), pos=n(N, C, k=0.5), w1=n(C, k=0.2, m=1.0), b1=n(C, k=0.2), W1=n(C, hidden, k=C ** -0.5), c1=n(hidden, k=0.1),
                      W2=n(hidden, C, k=hidden ** -0.5), c2=n(C, k=0.1), post_w=n(C, k=0.2, m=1.0), post_b=n(C, k=0.1), gate=n(B, C, k=0.3, m=0.5),
                      w2=n(C, k=0.2, m=1.0), b2=n(C, k=0.1), W3=n(C, hidden, k=C ** -0.5), c3=n(hidden, k=0.1))
        for k in ("table", "pos", "W1", "W2", "W3", "gate"):
            self.p[k] = self.p[k].to(self.dt)
        self.ids = torch.randint(0, V, (M,), device="cuda", generator=g).int()
        self.ids[::17] = -1
        self.places = (torch.arange(M, device="cuda") % N).int()
        self.dOut, self.dEnd = n(M, hidden).to(self.dt), n(M, C).to(self.dt)
        self.K = B * sbp.sbp_keep_count(sbp.SBP_MASK_RANDOM, N, 1, ratio)
        self.rows, self.offs = torch.empty(self.K, dtype=torch.int32, device="cuda"), torch.empty(B + 1, dtype=torch.int32, device="cuda")
        new = lambda r, c: torch.full((r, c), float("nan"), dtype=self.dt, device="cuda")
        for name, r, c in (("X", M, C), ("Z1", M, C), ("A", M, hidden), ("Y", M, C), ("R", M, C), ("Z2", M, C), ("out", M, hidden), ("dH", M, C),
                           ("dX", M, C), ("X_keep", self.K, C), ("Z1_keep", self.K, C), ("A_keep", self.K, hidden), ("Y_keep", self.K, C),
                           ("R_keep", self.K, C), ("Z2_keep", self.K, C), ("dZ2", self.K, C), ("dY", self.K, C), ("dA", self.K, hidden), ("dZ1", self.K, C)):
            setattr(self, name, new(r, c))
        self.g = {k: torch.full(v.shape, float("nan"), device="cuda") for k, v in self.p.items()}
        need = [sbp.sbp_linear_backward_workspace_bytes(self.code, M, self.K, a, b) for a, b in ((C, hidden), (hidden, C))]
        need += [sbp.sbp_block_norm_backward_workspace_bytes(self.code, M, self.K, C)]
        need += [sbp.sbp_embedding_backward_workspace_bytes(self.code, M, v, C) for v in (V, N)]
        need += [sbp.sbp_orthogonalize_workspace_bytes(self.code, 1, C, hidden)]
        self.ws = torch.full((max(need),), 255, dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.momentum, self.update = torch.zeros((C, hidden), device="cuda"), new(C, hidden)

    def linear_back(self, X_keep, dY, W, dW, db, dX, ci, co, flags):
        sbp.sbp_linear_backward(self.code, X_keep, dY, W, self.rows, None, self.M, self.K, ci, co, dW, db, dX, flags | sbp.SBP_FLAG_DX_COMPACT, self.ws,
                                self.ws.numel(), self.status)

    def run(self):
        p, g, M, K, C, H = self.p, self.g, self.M, self.K, self.C, self.hidden
        sbp.sbp_sample_keep(sbp.SBP_MASK_RANDOM, self.B, self.N, 1, self.K / M, 3, 0, 0, 0, self.rows, self.offs)
        sbp.sbp_embedding_forward(self.code, p["pos"], self.N, C, self.places, M, 1.0, None, self.X, self.status)
        sbp.sbp_embedding_forward(self.code, p["table"], self.V, C, self.ids, M, 2.0, self.X, self.X, self.status)
        sbp.sbp_block_norm_forward(self.code, self.kind, self.X, None, None, None, None, 1, 1.0, p["w1"], p["b1"], EPS, M, C, None, self.Z1, self.rows, None,
                                   K, None, self.X_keep, self.Z1_keep, self.status)
        sbp.sbp_linear_forward(self.code, self.Z1, p["W1"], p["c1"], M, C, H, self.A, flags=0, status_word=self.status)
        sbp.sbp_linear_forward(self.code, self.A, p["W2"], p["c2"], M, H, C, self.Y, self.rows, None, K, self.A_keep, 0, self.status)
        sbp.sbp_block_norm_forward(self.code, self.kind, self.X, self.Y, p["post_w"], p["post_b"], p["gate"], self.N, 0.8, p["w2"], p["b2"], EPS, M, C, self.R,
                                   self.Z2, self.rows, None, K, self.Y_keep, self.R_keep, self.Z2_keep, self.status)
        sbp.sbp_linear_forward(self.code, self.Z2, p["W3"], p["c3"], M, C, H, self.out, flags=0, status_word=self.status)
        # back: the loss is sum(dOut out) on the kept rows and sum(dEnd R) on all
        self.linear_back(self.Z2_keep, self.dOut, p["W3"], g["W3"], g["c3"], self.dZ2, C, H, 0)
        sbp.sbp_block_norm_backward(self.code, self.kind, self.dEnd, self.dZ2, self.R_keep, self.Y_keep, p["post_w"], p["post_b"], p["gate"], self.N, 0.8,
                                    p["w2"], EPS, self.rows, None, M, K, C, self.dH, self.dY, g["post_w"], g["post_b"], g["gate"], g["w2"], g["b2"], 0,
                                    self.ws, self.ws.numel(), self.status)
        # (the keep set is the block's: the gradient stays packed through its two layers)
        self.linear_back(self.A_keep, self.dY, p["W2"], g["W2"], g["c2"], self.dA, H, C, sbp.SBP_FLAG_DY_COMPACT)
        self.linear_back(self.Z1_keep, self.dA, p["W1"], g["W1"], g["c1"], self.dZ1, C, H, sbp.SBP_FLAG_DY_COMPACT)
        sbp.sbp_block_norm_backward(self.code, self.kind, self.dH, self.dZ1, self.X_keep, None, None, None, None, 1, 1.0, p["w1"], EPS, self.rows, None, M, K,
                                    C, self.dX, None, None, None, None, g["w1"], g["b1"], 0, self.ws, self.ws.numel(), self.status)
        sbp.sbp_embedding_backward(self.code, self.dX, self.ids, None, None, M, M, self.V, C, 2.0, g["table"], 0, self.ws, self.ws.numel(), self.status)
        sbp.sbp_embedding_backward(self.code, self.dX, self.places, None, None, M, M, self.N, C, 1.0, g["pos"], 0, self.ws, self.ws.numel(), self.status)
        sbp.sbp_orthogonalize(self.code, g["W1"], self.momentum, 0.9, 1, C, H, 5, 1e-7, 1.0, self.update, sbp.SBP_FLAG_NESTEROV, self.ws, self.ws.numel(),
                              self.status)

    def norm64(self, x, w, b):
        x = x - x.mean(1, keepdim=True) if self.kind == sbp.SBP_NORM_LAYER else x
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * w + b

    def reference(self):
        p = {k: v.double().requires_grad_() for k, v in self.p.items()}
        mask = torch.zeros(self.M, 1, device="cuda", dtype=torch.float64)
        mask[self.rows.long()] = 1.0
        kept = lambda x: x * mask + (x * (1 - mask)).detach()          # its gradient on the kept rows only
        known = (self.ids >= 0).double()[:, None]
        X = p["pos"][self.places.long()] + 2.0 * p["table"][self.ids.long().clamp_min(0)] * known
        Y = (self.norm64(X, p["w1"], p["b1"]) @ p["W1"] + p["c1"]) @ p["W2"] + p["c2"]
        R = 0.8 * X + kept(p["gate"].repeat_interleave(self.N, 0) * self.norm64(Y, p["post_w"], p["post_b"]))
        out = kept(self.norm64(R, p["w2"], p["b2"]) @ p["W3"] + p["c3"])
        loss = (out * self.dOut.double()).sum() + (R * self.dEnd.double()).sum()
        grads = dict(zip(p, torch.autograd.grad(loss, list(p.values()))))
        return R.detach(), out.detach(), grads


def rel(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,N,C,hidden,V,kind", [(4, 33, 64, 128, 50, 0), (3, 50, 192, 320, 700, 1), (16, 196, 768, 256, 30, 0), (1, 1, 64, 64, 3, 1)])
def test_a_training_step(dtype, B, N, C, hidden, V, kind):
    s = Step(dtype, B, N, C, hidden, V, kind)
    s.run()
    torch.cuda.synchronize()
    assert s.status.item() == 0
    R, out, grads = s.reference()
    assert rel(s.R, R) <= 5 * s.tol and rel(s.out, out) <= 7 * s.tol
    for k, want in grads.items():
        if want.norm() == 0:
            assert not s.g[k].any(), k
        else:
            assert rel(s.g[k], want) <= 8 * s.tol, (k, rel(s.g[k], want))
    # the update is that of the gradient which the step made
    U = 1.9 * s.g["W1"].double()                        # G + 0.9 (0.9 * 0 + G)
    X = U / (U.norm() + 1e-7)
    X = X.mT if C > hidden else X
    for _ in range(5):
        A = X @ X.mT
        X = 3.4445 * X + (-4.7750 * A + 2.0315 * A @ A) @ X
    X = X.mT if C > hidden else X
    # (a gradient of few rows has few directions: what is left of its roundings, 2^-23, grows by a factor 3.4445 a step in the others)
    assert rel(s.update, X) <= max(s.tol, 1e-4)
    assert torch.equal(s.momentum, s.g["W1"])


def test_the_step_captured_and_replayed_gives_the_same_bits():
    s = Step("bf16", 4, 65, 256, 512, 100, 0)
    s.run()
    torch.cuda.synchronize()
    names = ["R", "out", "dH", "dX", "update"]
    want = {n: getattr(s, n).clone() for n in names} | {k: v.clone() for k, v in s.g.items()}
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        s.run()
    for _ in range(2):
        for n in names:
            getattr(s, n).fill_(float("nan"))
        for v in s.g.values():
            v.fill_(float("nan"))
        s.momentum.zero_()
        s.ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert s.status.item() == 0
        for n in names:
            assert torch.equal(getattr(s, n), want[n]), n
        for k, v in s.g.items():
            assert torch.equal(v, want[k]), k
