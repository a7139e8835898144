"""A gated layer, the scores of a vocabulary and learning from a teacher, as a language model uses them: both projections of a gated
feed-forward block with the activation and the product of the two (and the block's gradients), log probabilities of given tokens with entropy
and the most likely alternatives, and the distillation loss against a teacher's top entries (and its gradient).  No logits are kept.

`run` computes each in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, where `own` is true,
through the binding's entry points.  Shapes are the benchmark's width of 768 with a gated block's inner width of 8/3 of it and a byte-pair
vocabulary, or generic ones; all inputs are drawn on the GPU from the seed alone."""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
IGNORE = -100


def _case(name, **c):
    return dict(c, name=name) if name else c


def _gated(name, dtype, out, M, N, K, tb=0, act="silu", bias=False, keep=False):
    return _case(name, kind="gated", dtype=dtype, out=out, M=M, N=N, K=K, tb=tb, act=act, bias=bias, keep=keep)


def _gated_grad(name, dtype, M, N, K, tb=0, act="silu"):
    return _case(name, kind="gated_grad", dtype=dtype, M=M, N=N, K=K, tb=tb, act=act)


def _score(name, dtype, T, V, D, top, scale=1.0):
    return _case(name, kind="score", dtype=dtype, T=T, V=V, D=D, top=top, scale=scale)


def _teach(name, dtype, T, V, D, k, scale=1.0, normalize=True):
    return _case(name, kind="teach", dtype=dtype, T=T, V=V, D=D, k=k, scale=scale, normalize=normalize)


def _teach_grad(name, dtype, T, V, D, k, scale=1.0, normalize=True):
    return _case(name, kind="teach_grad", dtype=dtype, T=T, V=V, D=D, k=k, scale=scale, normalize=normalize)


def listed():
    return [
        # a generated token's gated layer: 6 MB of weights, a matter of latency
        _gated("gated_one_token_bf16", "bf16", "bf16", 1, 2048, 768, tb=1),
        # a training batch's, both projections' results kept for the gradient
        _gated("gated_train_f16", "f16", "f16", 8192, 2048, 768, keep=True),
        # a prompt through a wider model's
        _gated("gated_prompt_bf16", "bf16", "bf16", 2048, 5632, 2048, tb=1, act="gelu"),
        # odd sizes in fp32, with biases
        _gated("gated_ragged_f32", "f32", "f32", 517, 803, 301, tb=1, act="relu", bias=True),
        # the whole block's gradients: of its input and of its three matrices
        _gated_grad("gated_grad_bf16", "bf16", 8192, 2048, 768),
        _gated_grad("gated_grad_ragged_f32", "f32", 333, 547, 205, tb=1, act="gelu"),
        # a generated token with its five most likely alternatives
        _score("score_one_token_bf16", "bf16", 1, 50257, 768, 5),
        # a teacher's, or a sampler's, batch: the log probability of each token, the entropy, eight alternatives
        _score("score_batch_f16", "f16", 4096, 50257, 768, 8),
        # an odd vocabulary in fp32 at a temperature of 0.7
        _score("score_ragged_f32", "f32", 301, 5003, 205, 20, scale=1.0 / 0.7),
        # the loss of a training batch against a teacher's sixteen most likely entries
        _teach("teach_f16", "f16", 4096, 50257, 768, 16),
        # its gradient, of the activations and of the vocabulary's weights
        _teach_grad("teach_grad_bf16", "bf16", 4096, 50257, 768, 16),
        # an odd vocabulary in fp32 at a temperature of 2, the teacher's probabilities as they are
        _teach_grad("teach_grad_ragged_f32", "f32", 333, 5003, 205, 7, scale=0.5, normalize=False),
    ]


def _logint(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: whole vectors as a rule, now and then any number."""
    n = _logint(rng, lo, hi)
    return n if rng.random() < 0.25 else max(lo, n // 8 * 8)


def draw(rng):
    kind = rng.choice(["gated", "gated", "gated_grad", "score", "score", "teach", "teach_grad"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    if kind in ("gated", "gated_grad"):
        most = 3.0e11 if dtype != "f32" else 3.0e10
        d = _width(rng, 64, 2048 if dtype != "f32" else 768)
        n = 8 * d // 3 if rng.random() < 0.25 else max(8, 8 * d // 3 // 8 * 8)
        each = (4.0 if kind == "gated" else 12.0) * n * d
        rows = max(1, min(_logint(rng, 1, 8192), int(most / each)))
        act, tb = rng.choice(["silu", "silu", "gelu", "relu", "none"]), rng.randint(0, 1)
        if kind == "gated_grad":
            return _gated_grad(None, dtype, rows, n, d, tb=tb, act=act)
        return _gated(None, dtype, rng.choice([dtype, dtype, "f32"]), rows, n, d, tb=tb, act=act, bias=rng.random() < 0.4, keep=rng.random() < 0.5)
    tokens, d, vocab = _logint(rng, 1, 4096 if dtype != "f32" else 512), _width(rng, 64, 1024), _logint(rng, 1000, 52000)
    most = 9.0e11 if dtype != "f32" else 1.0e11
    tokens = max(1, min(tokens, int(most / (6.0 * vocab * d))))
    scale = rng.choice([1.0, 1.0, 0.5, 1.0 / 0.7])
    if kind == "score":
        return _score(None, dtype, tokens, vocab, d, rng.choice([0, 1, _logint(rng, 2, 32), _logint(rng, 2, 32)]), scale)
    make = _teach if kind == "teach" else _teach_grad
    return make(None, dtype, tokens, vocab, d, _logint(rng, 1, 64), scale, rng.random() < 0.6)


# ---------------------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, out = TORCH[case["dtype"]], TORCH[case.get("out", case["dtype"])]

    def normal(shape, sigma=1.0, grid=None):
        t = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, sigma, generator=g)
        return (t if grid is None else torch.round(t / grid) * grid).to(dt)

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = {"case": case}
    if case["kind"] in ("gated", "gated_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        s["x"] = normal((M, K))
        # both projections side by side in one matrix, as checkpoints hold them: [K][gate N, up N], or its transpose
        s["w"] = normal((2 * N, K) if case["tb"] else (K, 2 * N), 1.0 / math.sqrt(K))
        if case["kind"] == "gated":
            s["bias"] = normal((2, N), 0.5) if case["bias"] else None
            s["z"] = empty((M, 2 * N), out) if case["keep"] else None
            s["y"] = empty((M, N), out)
        else:
            s["down"], s["z"], s["dy"] = normal((N, K), 1.0 / math.sqrt(N)), normal((M, 2 * N)), normal((M, K))
            s["dz"], s["h"], s["dx"] = empty((M, 2 * N), dt), empty((M, N), dt), empty((M, K), dt)
            s["dw"], s["ddown"] = empty(tuple(s["w"].shape), dt), empty((N, K), dt)
        return s
    T, V, D = case["T"], case["V"], case["D"]
    sigma = 2.0 / math.sqrt(D)
    # Values on a grid, as quantised ones are: the products sum exactly in 32 bits in any order, so which entries are the largest is the same for
    # every way of computing them.
    s["x"] = normal((T, D), grid=1.0 / 16)
    s["w"] = normal((V, D), sigma, grid=2.0 ** math.floor(math.log2(sigma)) / 32)
    if case["kind"] == "score":
        targets = torch.randint(0, V, (T,), generator=g, device="cuda")
        if T > 1:                            # a twentieth of a batch is padding
            targets[rand(T) < 0.05] = IGNORE
        s["targets"] = targets
        s["logprob"], s["entropy"] = empty((T,), torch.float32), empty((T,), torch.float32)
        s["top_index"], s["top_logprob"] = empty((T, case["top"]), torch.int64), empty((T, case["top"]), torch.float32)
        return s
    # a teacher's entries: distinct, falling probabilities; fewer of them for some tokens, none for padding (a twentieth of a batch)
    k = case["k"]
    gap = 1 + (rand(T, k) * (V // k)).long().clamp(max=V // k - 1)
    s["index"] = (torch.randint(0, V, (T, 1), generator=g, device="cuda") + gap.cumsum(1)) % V
    fall = torch.cumsum(-torch.log(1.0 - 0.999 * rand(T, k)), 1)
    s["teacher"] = -fall - torch.log(torch.exp(-fall).sum(1, keepdim=True) / (0.5 + 0.49 * rand(T, 1)))
    there = torch.where(rand(T) < 0.9, k, torch.randint(1, k + 1, (T,), generator=g, device="cuda"))
    if T > 1:
        there = torch.where(rand(T) < 0.05, 0, there)
    s["index"] = torch.where(torch.arange(k, device="cuda") < there[:, None], s["index"], -1)
    s["lse"] = empty((T,), torch.float32)
    if case["kind"] == "teach":
        s["loss"] = empty((T,), torch.float32)
    else:
        s["lse"] = torch.logsumexp((s["x"].float() @ s["w"].float().t()) * case["scale"], 1)
        # the mean over the tokens, times the loss scale that training in f16 uses
        s["dloss"] = torch.full((T,), (4096.0 if case["dtype"] == "f16" else 1.0) / T, device="cuda")
        s["dx"], s["dw"] = empty((T, D), dt), empty((V, D), dt)
    return s


# ---------------------------------------------------------------------------------------------------------------------
GELU_C = math.sqrt(2.0 / math.pi)


def _act(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(GELU_C * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        t = torch.tanh(GELU_C * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * GELU_C * (1.0 + 3.0 * 0.044715 * z * z)
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 + z * (1.0 - e))
    return torch.ones_like(z)


def _largest(z, n):
    """The n largest of each row, equal ones from the lowest index: sorted by one whole number, the value's order in front of the index's."""
    bits = z.view(torch.int32).long()
    order = torch.where(bits < 0, -1 - (bits & 0x7FFFFFFF), bits)
    key = order * 2 ** 32 + (2 ** 32 - 1 - torch.arange(z.shape[1], device=z.device))
    at = 2 ** 32 - 1 - (key.topk(n, 1).values & 0xFFFFFFFF)
    return at, z.gather(1, at)


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind in ("gated", "gated_grad"):
        N, x = case["N"], s["x"].float()
        w = s["w"].float().t() if case["tb"] else s["w"].float()
        if kind == "gated":
            out = TORCH[case["out"]]
            z = x @ w
            if s["bias"] is not None:
                z = z + s["bias"].float().reshape(-1)
            y = _act(z[:, :N], case["act"]) * z[:, N:]
            return {"y": y.to(out), "z": z.to(out) if case["keep"] else None}
        dt, dy = TORCH[case["dtype"]], s["dy"].float()
        gate, up = s["z"][:, :N].float(), s["z"][:, N:].float()
        d = dy @ s["down"].float().t()
        # (what the pass hands on between its products is of the type, as the layer's values are)
        h = (_act(gate, case["act"]) * up).to(dt)
        dz = torch.cat([d * up * _act_slope(gate, case["act"]), d * _act(gate, case["act"])], 1).to(dt)
        dw = x.t() @ dz.float()
        return {"dz": dz, "dx": (dz.float() @ w.t()).to(dt), "dw": (dw.t() if case["tb"] else dw).to(dt).contiguous(), "ddown": (h.float().t() @ dy).to(dt)}
    z = s["x"].float() @ s["w"].float().t()
    if case["scale"] != 1.0:
        z = z * case["scale"]
    if kind == "score":
        t = s["targets"]
        counts = t != IGNORE
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - top)
        total = e.sum(1)
        rest = torch.log(total)
        at = z.gather(1, torch.where(counts, t, torch.zeros_like(t))[:, None])[:, 0]
        entropy = rest - (e * (z - top)).sum(1) / total
        index, value = _largest(z, case["top"])
        return {"logprob": torch.where(counts, (at - top[:, 0]) - rest, torch.zeros_like(at)), "entropy": entropy, "top_index": index,
                "top_logprob": (value - top) - rest[:, None]}
    there = s["index"] >= 0
    at = torch.where(there, s["index"], torch.zeros_like(s["index"]))
    q = s["teacher"]
    if case["normalize"]:
        q = torch.where(there, q * case["scale"], torch.full_like(q, -1e30))
        q = q - q.amax(1, keepdim=True)
        q = q - torch.log(torch.exp(q).sum(1, keepdim=True))
    p = torch.where(there, torch.exp(q), torch.zeros_like(q))
    mass = p.sum(1)
    if kind == "teach":
        top = z.amax(1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
        loss = (p * (torch.where(there, q, torch.zeros_like(q)) - z.gather(1, at))).sum(1) + mass * lse
        return {"loss": loss, "lse": lse}
    g = torch.exp(z - s["lse"][:, None]) * mass[:, None]
    g = g.scatter_add(1, at, -p) * (s["dloss"] * case["scale"])[:, None]
    return {"dx": (g @ s["w"].float()).to(s["dx"].dtype), "dw": (g.t() @ s["x"].float()).to(s["dw"].dtype)}


def _kept(s, name, make):
    """What a program makes once for its buffers and keeps: problems and workspaces."""
    if name not in s:
        s[name] = make()
    return s[name]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def _pair(t, width):
    """[rows][2 width] as two matrices."""
    return t.view(t.shape[0], 2, width).transpose(0, 1)


def _own(s):
    from paper_2502_11407_amd import binding as gs
    case = s["case"]
    kind, dtype = case["kind"], case["dtype"]
    if kind in ("gated", "gated_grad"):
        M, N, K, tb = case["M"], case["N"], case["K"], case["tb"]
        if kind == "gated":
            p = _kept(s, "p", lambda: gs.gemm_problem(dtype, M, N, K, transB=tb, out_dtype=case["out"]))
            w = s["w"].view(2, N, K) if tb else _pair(s["w"], N)
            gs.gated_gemm(p, s["x"], w, s["y"], act=case["act"], bias=s["bias"], preact=_pair(s["z"], N) if case["keep"] else None)
            return {"y": s["y"], "z": s["z"]}
        back = _kept(s, "back", lambda: gs.gemm_problem(dtype, M, N, K, transB=1, out_dtype=dtype))
        of_x = _kept(s, "of_x", lambda: gs.gemm_problem(dtype, M, K, 2 * N, transB=1 - tb, out_dtype=dtype))
        of_w = _kept(s, "of_w", lambda: gs.gemm_problem(dtype, 2 * N if tb else K, K if tb else 2 * N, M, transA=1, out_dtype=dtype))
        of_down = _kept(s, "of_down", lambda: gs.gemm_problem(dtype, N, K, M, transA=1, out_dtype=dtype))
        ws = _kept(s, "ws", lambda: _bytes(max(gs.gemm_fused_workspace_bytes(p) for p in (of_x, of_w, of_down))))
        gs.gated_act_grad(back, s["dy"], s["down"], _pair(s["z"], N), _pair(s["dz"], N), act=case["act"], H=s["h"])
        gs.gemm_fused(of_x, s["dz"], s["w"], s["dx"], workspace=ws)
        gs.gemm_fused(of_w, s["dz"] if tb else s["x"], s["x"] if tb else s["dz"], s["dw"], workspace=ws)
        gs.gemm_fused(of_down, s["h"], s["dy"], s["ddown"], workspace=ws)
        return {"dz": s["dz"], "dx": s["dx"], "dw": s["dw"], "ddown": s["ddown"]}
    T, V, D = case["T"], case["V"], case["D"]
    if kind == "score":
        ws = _kept(s, "ws", lambda: _bytes(gs.logprobs_workspace_bytes(dtype, T, V, D, case["top"])))
        tops = {"top_index": s["top_index"], "top_logprob": s["top_logprob"]} if case["top"] else {}
        gs.logprobs(s["x"], s["w"], targets=s["targets"], logprob=s["logprob"], entropy=s["entropy"], scale=case["scale"], ignore_index=IGNORE, workspace=ws, **tops)
        return {"logprob": s["logprob"], "entropy": s["entropy"], "top_index": s["top_index"], "top_logprob": s["top_logprob"]}
    if kind == "teach":
        ws = _kept(s, "ws", lambda: _bytes(gs.distill_workspace_bytes(dtype, T, V, D, case["k"])))
        gs.distill_forward(s["x"], s["w"], s["index"], s["teacher"], s["loss"], s["lse"], scale=case["scale"], normalize=case["normalize"], workspace=ws)
        return {"loss": s["loss"], "lse": s["lse"]}
    ws = _kept(s, "ws", lambda: _bytes(gs.distill_workspace_bytes(dtype, T, V, D, case["k"], backward=True)))
    gs.distill_backward(s["x"], s["w"], s["index"], s["teacher"], s["lse"], s["dloss"], s["dx"], s["dw"], scale=case["scale"], normalize=case["normalize"], workspace=ws)
    return {"dx": s["dx"], "dw": s["dw"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], BYTES[case["dtype"]]
    if kind in ("gated", "gated_grad"):
        M, N, K = case["M"], case["N"], case["K"]
        if kind == "gated":
            return {"bytes": (M * K + 2 * K * N + 2 * N * int(case["bias"])) * e + (3 if case["keep"] else 1) * M * N * BYTES[case["out"]], "flops": 4.0 * M * N * K}
        # x, dy, z and the three matrices in; the same again as gradients, and dz
        return {"bytes": (2 * M * K + 2 * M * N + 3 * K * N + M * K + 2 * M * N + 3 * K * N) * e, "flops": 12.0 * M * N * K}
    T, V, D = case["T"], case["V"], case["D"]
    if kind == "score":
        return {"bytes": (T * D + V * D) * e + T * (16 + 12 * case["top"]), "flops": 2.0 * T * V * D}
    if kind == "teach":
        return {"bytes": (T * D + V * D) * e + T * (8 + 12 * case["k"]), "flops": 2.0 * T * V * D}
    return {"bytes": 2 * (T * D + V * D) * e + T * (8 + 12 * case["k"]), "flops": 6.0 * T * V * D}


# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    """The definitions in 64 bits, differentiated by autograd where a gradient is asked for."""
    s = prepare(case, seed)
    kind = case["kind"]
    f = torch.nn.functional
    acts = {"none": lambda z: z, "relu": f.relu, "gelu": lambda z: f.gelu(z, approximate="tanh"), "silu": f.silu}
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    if kind in ("gated", "gated_grad"):
        weights = d["w"] if case["tb"] else d["w"].mT
        if kind == "gated":
            z = f.linear(d["x"], weights, None if s["bias"] is None else d["bias"].flatten())
            gate, up = z.chunk(2, 1)
            return {"y": acts[case["act"]](gate) * up, "z": z if case["keep"] else None}
        z, down = d["z"].requires_grad_(True), d["down"].requires_grad_(True)
        gate, up = z.chunk(2, 1)
        torch.matmul(acts[case["act"]](gate) * up, down).backward(d["dy"])
        # (the input's and the weights' gradients go on from dz in the type where it is of 16 bits: those have no value of their own)
        if case["dtype"] != "f32":
            return {"dz": z.grad, "dx": None, "dw": None, "ddown": None}
        dw = torch.matmul(z.grad.mT, d["x"])
        return {"dz": z.grad, "dx": torch.matmul(z.grad, weights), "dw": dw if case["tb"] else dw.mT.contiguous(), "ddown": down.grad}
    if kind == "teach_grad":
        d["x"].requires_grad_(True)
        d["w"].requires_grad_(True)
    z = f.linear(d["x"], d["w"]) * case["scale"]
    logs = torch.log_softmax(z, 1)
    if kind == "score":
        logprob = -f.nll_loss(logs, s["targets"], ignore_index=IGNORE, reduction="none")
        return {"logprob": logprob, "entropy": torch.special.entr(logs.exp()).sum(1), "top_index": None,
                "top_logprob": torch.sort(logs, 1, descending=True).values[:, :case["top"]]}
    there = s["index"].ge(0)
    q = d["teacher"].masked_fill(~there, -math.inf)
    if case["normalize"]:
        q = torch.log_softmax(q * case["scale"], 1).masked_fill(~there, -math.inf)
    p = torch.exp(q)
    loss = torch.special.xlogy(p, p).sum(1) - (p * logs.gather(1, s["index"].clamp(min=0))).sum(1)
    if kind == "teach":
        return {"loss": loss.detach(), "lse": torch.logsumexp(z, 1).detach()}
    (loss * d["dloss"]).sum().backward()
    return {"dx": d["x"].grad, "dw": d["w"].grad}
