"""The most likely entries where logits are close to one another beside their size, as a common offset of a token's logits makes them: what a piece of the
vocabulary leaves in the workspace holds only the logits that may be among the largest, so nothing else in it may be taken for one.

The workspace is filled beforehand with a number above every logit: wherever it is read as a logit it wins.  Logits are on a grid of 2^-17 between 64 and 128, which
is fp32's own there, and sums of three multiples of it that have 6 bits each: every partial sum is exact in any order, in every type.  So which entries are the
largest is known.  Tolerance, u = 2^-24: the maximum is exact and what is left of the exponentials' arguments is below 2, so each term, the sums (64 roundings
one after the other at most) and log sum are off by 6e-6 together; lse and a log probability are rounded once more."""
import gc

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
KINDS = 7                                         # different distributions, token t has the t % KINDS'th


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()                                 # (other modules count the device memory that is in use)


def operands(dtype, T, V, spread, sign, seed, width=3 * KINDS + 1):
    """z[t][v] = sign * 100 + steps[v][t % KINDS] * 2^-17."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if spread == "even":                          # over a hundredth
        steps = torch.randint(0, 1311, (V, KINDS), generator=g, device="cuda")
    elif spread == "normal":                      # a tenth wide
        steps = (torch.empty((V, KINDS), device="cuda").normal_(131072.0, 13107.0, generator=g)).round().long().clamp(0, 262143)
    else:                                         # "few": nearly all are equal to many others
        steps = torch.randint(0, 6, (V, KINDS), generator=g, device="cuda")
    X, W = torch.zeros((T, width), device="cuda"), torch.zeros((V, width), device="cuda")
    X[:, 0], W[:, 0] = sign, 100.0
    for part in range(3):                         # (2^-10 of each part's size in X: both are normal numbers in every type)
        for kind in range(KINDS):
            X[kind::KINDS, 1 + 3 * kind + part] = 2.0 ** -10
            W[:, 1 + 3 * kind + part] = (steps[:, kind] // 64 ** part % 64).float() * 2.0 ** (6 * part - 7)
    return X.to(TORCH[dtype]), W.to(TORCH[dtype])


def fill(ws, value):
    ws.view(torch.float32).fill_(value)


def outputs(T, top):
    return {"lse": torch.full((T,), 7.0, device="cuda"), "top_index": torch.full((T, top), 7, dtype=torch.int64, device="cuda"),
            "top_logprob": torch.full((T, top), 7.0, device="cuda")}


def wanted(X, W, top):
    """By kinds: the first KINDS tokens are one of each."""
    z = X[:KINDS].double() @ W.double().t()
    assert bool((z.float().double() == z).all())
    best = torch.sort(z, dim=1, descending=True, stable=True)
    return best.indices[:, :top], best.values[:, :top], torch.logsumexp(z, 1)


def check(out, want):
    index, value, lse = want
    T = out["lse"].shape[0]
    kind = torch.arange(T, device="cuda") % KINDS
    wrong = (out["top_index"] != index[kind]).any(1)
    assert not bool(wrong.any()), "%d of %d tokens" % (int(wrong.sum()), T)
    lse, logs = lse[kind], (value - lse[:, None])[kind]
    assert bool(((out["lse"].double() - lse).abs() <= 6e-6 + 2 * U * lse.abs()).all())
    assert bool(((out["top_logprob"].double() - logs).abs() <= 6e-6 + 2 * U * logs.abs()).all())


@pytest.mark.parametrize("spread", ["even", "normal", "few"])
@pytest.mark.parametrize("T", [3, 200, 700, 1100])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_in_pieces(gs, dtype, T, spread):
    """With 8, 4 and 1 waves a token, on both sides of the count of alternatives that changes how the bar is found."""
    V = 12_007
    for sign in (1.0, -1.0):
        X, W = operands(dtype, T, V, spread, sign, T, 22 if sign > 0 else 24)         # (rows that are whole vectors, too)
        for top in (1, 8, 24, 40, 64):
            n = gs.logprobs_workspace_bytes(dtype, T, V, X.shape[1], top)
            want = wanted(X, W, top) if T >= KINDS else wanted(X.repeat(3, 1), W, top)
            if T < KINDS:
                want = tuple(w[:T] for w in want)
            for part in (4, 9):                   # at least so many pieces
                ws = torch.empty(n // part // 256 * 256, dtype=torch.uint8, device="cuda")
                fill(ws, 140.0 if sign > 0 else -70.0)
                out = outputs(T, top)
                gs.logprobs(X, W, workspace=ws, **out)
                check(out, want)


@pytest.mark.parametrize("T,V,top", [(640, 120_000, 8), (2100, 50_257, 8), (2100, 50_257, 33)])
def test_at_full_room(gs, T, V, top):
    for spread in ("even", "normal"):
        X, W = operands("bf16", T, V, spread, 1.0, 11, 32)
        ws = torch.empty(gs.logprobs_workspace_bytes("bf16", T, V, X.shape[1], top), dtype=torch.uint8, device="cuda")
        fill(ws, 140.0)
        out = outputs(T, top)
        gs.logprobs(X, W, workspace=ws, **out)
        check(out, wanted(X, W, top))


def test_after_a_call_of_larger_logits(gs):
    """One workspace for calls of a program, one after the other and in a graph."""
    T, V, top = 300, 12_007, 8
    X, W = operands("f16", T, V, "normal", 1.0, 3)
    n = gs.logprobs_workspace_bytes("f16", T, V, X.shape[1], top) // 5 // 256 * 256
    ws, out, want = torch.empty(n, dtype=torch.uint8, device="cuda"), outputs(T, top), wanted(X, W, top)
    larger, other = X * 2, outputs(T, top)
    call = lambda: gs.logprobs(X, W, workspace=ws, **out)
    before = lambda: gs.logprobs(larger, W, workspace=ws, **other)
    before()
    call()
    check(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        before()
        for v in out.values():
            v.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        check(out, want)
