"""A small student learns from a teacher's most likely entries, with gated layers, scores and the distillation loss of the binding:

    teacher: embedding -> gated block -> scores of the vocabulary: its top entries and their log probabilities
    student: embedding -> gated block -> distillation loss against them -> gradients of all of its matrices

Every product of the forward and the backward pass is one call of the binding; torch holds the tensors, gathers embeddings and applies the
updates.  Run: python examples/distill_step.py [f32|f16|bf16]  (needs an MI355X)."""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_11407_amd import binding as gs  # noqa: E402

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def room(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


class Model:
    """x = embed[token]; y = x + (silu(x Wg) * (x Wu)) Wd; logits = y head^T.  Both projections of the gated block lie side by side in one matrix."""

    def __init__(self, dtype="bf16", vocab=1009, width=128, inner=344, seed=0):
        self.dtype, self.vocab, self.width, self.inner = dtype, vocab, width, inner
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def normal(*shape, sigma):
            return torch.empty(shape, device="cuda").normal_(0.0, sigma, generator=g).to(TORCH[dtype])
        self.w = {"embed": normal(vocab, width, sigma=1.0), "both": normal(width, 2 * inner, sigma=width ** -0.5), "down": normal(inner, width, sigma=inner ** -0.5),
                  "head": normal(vocab, width, sigma=2 * width ** -0.5)}

    def empty(self, *shape):
        return torch.empty(shape, dtype=TORCH[self.dtype], device="cuda")

    def halves(self, t):
        """[rows][2 inner] as its two halves [2][rows][inner]."""
        return t.view(t.shape[0], 2, self.inner).transpose(0, 1)

    def product(self, A, B, transA=0, transB=0, **ends):
        M, K = (A.shape[1], A.shape[0]) if transA else A.shape
        N = B.shape[0] if transB else B.shape[1]
        p = gs.gemm_problem(self.dtype, M, N, K, transA, transB, out_dtype=self.dtype)
        out = self.empty(M, N)
        gs.gemm_fused(p, A, B, out, workspace=room(gs.gemm_fused_workspace_bytes(p)), **ends)
        return out

    def forward(self, tokens):
        """What the loss and the backward pass need."""
        w, T = self.w, tokens.shape[0]
        s = {"tokens": tokens, "x": w["embed"][tokens], "z": self.empty(T, 2 * self.inner), "h": self.empty(T, self.inner)}
        p = gs.gemm_problem(self.dtype, T, self.inner, self.width, out_dtype=self.dtype)
        gs.gated_gemm(p, s["x"], self.halves(w["both"]), s["h"], preact=self.halves(s["z"]))
        s["y"] = self.product(s["h"], w["down"], residual=s["x"])
        return s

    def scores(self, tokens, targets=None, top=8, scale=1.0):
        """Log probabilities of the targets, entropies, and the `top` most likely entries with theirs."""
        s, T = self.forward(tokens), tokens.shape[0]
        out = {"entropy": torch.empty(T, device="cuda"), "top_index": torch.empty((T, top), dtype=torch.int64, device="cuda"), "top_logprob": torch.empty((T, top), device="cuda")}
        if targets is not None:
            out["logprob"] = torch.empty(T, device="cuda")
        gs.logprobs(s["y"], self.w["head"], targets=targets, scale=scale, workspace=room(gs.logprobs_workspace_bytes(self.dtype, T, self.vocab, self.width, top)), **out)
        return out

    def loss(self, s, index, teacher, scale=1.0):
        T = s["y"].shape[0]
        s["loss"], s["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        ws = room(gs.distill_workspace_bytes(self.dtype, T, self.vocab, self.width, index.shape[1]))
        gs.distill_forward(s["y"], self.w["head"], index, teacher, s["loss"], s["lse"], scale=scale, workspace=ws)
        return s["loss"]

    def backward(self, s, index, teacher, dloss, scale=1.0):
        """Gradients of all weights, and of the gathered embeddings in the embedding's place."""
        w, T, g = self.w, s["x"].shape[0], {}
        dy, g["head"] = torch.empty_like(s["y"]), torch.empty_like(w["head"])
        ws = room(gs.distill_workspace_bytes(self.dtype, T, self.vocab, self.width, index.shape[1], backward=True))
        gs.distill_backward(s["y"], w["head"], index, teacher, s["lse"], dloss, dy, g["head"], scale=scale, workspace=ws)
        # the gradients of both projections' results take their place
        p = gs.gemm_problem(self.dtype, T, self.inner, self.width, transB=1, out_dtype=self.dtype)
        h, dz = self.empty(T, self.inner), s["z"]
        gs.gated_act_grad(p, dy, w["down"], self.halves(s["z"]), self.halves(dz), H=h)
        g["down"] = self.product(h, dy, transA=1)
        g["both"] = self.product(s["x"], dz, transA=1)
        dx = self.product(dz, w["both"], transB=1, residual=dy)
        g["embed"] = torch.zeros_like(w["embed"], dtype=torch.float32).index_add_(0, s["tokens"], dx.float()).to(dx.dtype)
        return g

    def step(self, tokens, index, teacher, rate):
        """One step of gradient descent on the mean loss; the loss before it."""
        s, T = self.forward(tokens), tokens.shape[0]
        loss = self.loss(s, index, teacher)
        scale = 1024.0 if self.dtype == "f16" else 1.0             # (loss scaling, undone in the update)
        g = self.backward(s, index, teacher, torch.full((T,), scale / T, device="cuda"))
        for name, grad in g.items():
            self.w[name].copy_(self.w[name].float() - rate / scale * grad.float())
        return loss.mean()


def main(dtype="bf16", steps=20):
    teacher, student = Model(dtype, inner=512, seed=1), Model(dtype, seed=2)
    tokens = torch.arange(500, device="cuda") * 2
    lesson = teacher.scores(tokens)
    losses = [float(student.step(tokens, lesson["top_index"], lesson["top_logprob"], 20.0)) for _ in range(steps)]
    print("loss", " ".join("%.3f" % v for v in losses))
    one = student.scores(tokens[3:4], targets=lesson["top_index"][3, :1], top=3)
    print("the teacher's first choice %.3f, entropy %.3f, alternatives %s" % (float(one["logprob"]), float(one["entropy"]), one["top_index"][0].tolist()))
    return losses


if __name__ == "__main__":
    main(*sys.argv[1:2])
