"""A small language model's training step and a token's score, with the products that are consumed where they are produced:

    embedding -> MLP block (bias, gelu and residual in the products) -> expert block (products grouped by expert) -> loss over the vocabulary

Every product of the forward and the backward pass is one call of the binding; torch holds the tensors, gathers embeddings, routes tokens and
applies the updates.  Run: python examples/lm_step.py [f32|f16|bf16]  (needs an MI355X)."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_11407_amd import binding as gs  # noqa: E402

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


class Model:
    """Weights are row-major [in][out]; the vocabulary's [entries][width] serve as embedding and as projection of their own."""

    def __init__(self, dtype="bf16", vocab=1009, width=128, experts=4, seed=0):
        self.dtype, self.vocab, self.width, self.experts = dtype, vocab, width, experts
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape, sigma):
            return torch.empty(shape, device="cuda").normal_(0.0, sigma, generator=g).to(TORCH[dtype])
        D, H, E = width, 4 * width, experts
        self.w = {"embed": normal(vocab, D, sigma=1.0), "router": normal(D, E, sigma=D ** -0.5),
                  "up": normal(D, H, sigma=D ** -0.5), "up_bias": normal(H, sigma=0.1), "down": normal(H, D, sigma=0.5 * H ** -0.5), "down_bias": normal(D, sigma=0.1),
                  "e_up": normal(E, D, H, sigma=D ** -0.5), "e_up_bias": normal(E, H, sigma=0.1), "e_down": normal(E, H, D, sigma=0.5 * H ** -0.5),
                  "e_down_bias": normal(E, D, sigma=0.1), "head": normal(vocab, D, sigma=D ** -0.5)}

    def empty(self, *shape):
        return torch.empty(shape, dtype=TORCH[self.dtype], device="cuda")

    def _product(self, A, B, out=None, transA=0, transB=0, grad_at=None, **ends):
        M, K = (A.shape[1], A.shape[0]) if transA else A.shape
        N = B.shape[0] if transB else B.shape[1]
        p = gs.gemm_problem(self.dtype, M, N, K, transA, transB, out_dtype=self.dtype)
        out = self.empty(M, N) if out is None else out
        n = gs.gemm_fused_workspace_bytes(p)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        if grad_at is not None:
            gs.gemm_act_grad(p, A, B, grad_at, out, "gelu", workspace=ws)
        else:
            gs.gemm_fused(p, A, B, out, workspace=ws, **ends)
        return out

    def _experts(self, A, B, offsets, transB=0, grad_at=None, **ends):
        N, K = (B.shape[1], B.shape[2]) if transB else (B.shape[2], B.shape[1])
        p = gs.grouped_problem(self.dtype, self.experts, A.shape[0], N, K, transB, self.dtype)
        out = self.empty(A.shape[0], N)
        if grad_at is not None:
            gs.grouped_act_grad(p, offsets, A, B, grad_at, out, "gelu")
        else:
            gs.grouped_gemm(p, offsets, A, B, out, **ends)
        return out

    def _column_sums(self, d, like, offsets=None):
        out = torch.empty_like(like)
        n = gs.bias_grad_workspace_bytes(1 if offsets is None else self.experts, d.shape[0], d.shape[1], self.dtype)
        gs.bias_grad(d, out, offsets=offsets, workspace=torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
        return out

    def forward(self, tokens, targets):
        """Everything the backward pass needs; `loss` and `lse` are in the order of the sorted tokens, `order`."""
        w, T = self.w, tokens.shape[0]
        s = {"tokens": tokens, "x": w["embed"][tokens]}
        s["z"] = self.empty(T, 4 * self.width)
        s["h"] = self._product(s["x"], w["up"], bias=w["up_bias"], act="gelu", preact=s["z"])
        s["x1"] = self._product(s["h"], w["down"], bias=w["down_bias"], residual=s["x"])
        # each token goes to its highest-scoring expert; rows sorted by expert, the experts' offsets stay on the device
        expert = (s["x1"].float() @ w["router"].float()).argmax(1)
        s["order"] = torch.argsort(expert, stable=True)
        counts = torch.zeros(self.experts, dtype=torch.int64, device="cuda").scatter_add_(0, expert, torch.ones_like(expert))
        s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).int()
        s["xs"] = s["x1"][s["order"]]
        s["ez"] = self.empty(T, 4 * self.width)
        s["eh"] = self._experts(s["xs"], w["e_up"], s["offsets"], bias=w["e_up_bias"], act="gelu", preact=s["ez"])
        s["x2"] = self._experts(s["eh"], w["e_down"], s["offsets"], bias=w["e_down_bias"], residual=s["xs"])
        s["targets"] = targets[s["order"]]
        s["loss"], s["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        ws = torch.empty(gs.xent_workspace_bytes(self.dtype, T, self.vocab, self.width), dtype=torch.uint8, device="cuda")
        gs.xent_forward(s["x2"], w["head"], s["targets"], s["loss"], s["lse"], workspace=ws)
        return s

    def backward(self, s, dloss):
        """Gradients of all weights but the router's (the choice of an expert has none)."""
        w, T, off, g = self.w, s["x"].shape[0], s["offsets"], {}
        dx2, g["head"] = torch.empty_like(s["x2"]), torch.empty_like(w["head"])
        ws = torch.empty(gs.xent_workspace_bytes(self.dtype, T, self.vocab, self.width, backward=True), dtype=torch.uint8, device="cuda")
        gs.xent_backward(s["x2"], w["head"], s["targets"], s["lse"], dloss, dx2, g["head"], workspace=ws)
        g["e_down_bias"] = self._column_sums(dx2, w["e_down_bias"], off)
        g["e_down"] = torch.empty_like(w["e_down"])
        gs.grouped_wgrad(gs.grouped_problem(self.dtype, self.experts, T, self.width, 4 * self.width, 0, self.dtype), off, s["eh"], dx2, g["e_down"])
        dez = self._experts(dx2, w["e_down"], off, transB=1, grad_at=s["ez"])
        g["e_up_bias"] = self._column_sums(dez, w["e_up_bias"], off)
        g["e_up"] = torch.empty_like(w["e_up"])
        gs.grouped_wgrad(gs.grouped_problem(self.dtype, self.experts, T, 4 * self.width, self.width, 0, self.dtype), off, s["xs"], dez, g["e_up"])
        dxs = self._experts(dez, w["e_up"], off, transB=1, residual=dx2)
        dx1 = torch.empty_like(dxs)
        dx1[s["order"]] = dxs
        g["down_bias"] = self._column_sums(dx1, w["down_bias"])
        g["down"] = self._product(s["h"], dx1, transA=1)
        dz = self._product(dx1, w["down"], transB=1, grad_at=s["z"])
        g["up_bias"] = self._column_sums(dz, w["up_bias"])
        g["up"] = self._product(s["x"], dz, transA=1)
        dx = self._product(dz, w["up"], transB=1, residual=dx1)
        g["embed"] = torch.zeros_like(w["embed"], dtype=torch.float32).index_add_(0, s["tokens"], dx.float()).to(dx.dtype)
        return g

    def step(self, tokens, targets, rate):
        """One step of gradient descent; the mean loss before it."""
        s = self.forward(tokens, targets)
        count = (targets != -100).sum().clamp(min=1)
        scale = 1024.0 if self.dtype == "f16" else 1.0             # (loss scaling, undone in the update)
        g = self.backward(s, torch.full_like(s["loss"], 1.0) * scale / count)
        for name, grad in g.items():
            self.w[name].copy_(self.w[name].float() - rate / scale * grad.float())
        return s["loss"].sum() / count

    def score(self, token, target):
        """Negative log-likelihood of one token after another: the same calls on a single row."""
        return self.forward(token.view(1), target.view(1))["loss"][0]


def main(dtype="bf16", steps=20):
    m = Model(dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    tokens = torch.randint(0, m.vocab, (500,), generator=g, device="cuda")
    targets = (tokens * 7 + 3) % m.vocab                            # something that can be learnt
    targets[::50] = -100                                            # padding
    losses = [float(m.step(tokens, targets, 1.0)) for _ in range(steps)]
    print("loss", " ".join("%.3f" % v for v in losses))
    print("score of one token %.3f" % float(m.score(tokens[1], targets[1])))
    return losses


if __name__ == "__main__":
    main(*sys.argv[1:2])
