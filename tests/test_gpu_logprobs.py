"""Scores of a vocabulary (log probabilities of given tokens, entropy and the most likely entries, logits never stored) against the definition
in 64 bits.

Operands are on grids on which every logit is a sum that fp32 holds exactly, so which entries are the largest, and which are equal, is known.  With
u = 2^-24: scale times a logit is rounded once (2 u |z|); lse is off by that and by the rounding of the exponentials' arguments (at most 100: 1e-5
relative at the very most, as the sum's terms; 4e-6 for the spreads here), of sums and joins (2e-6) and its own; log probabilities the same,
the entropy by the weights times the spread: 8e-6 (1 + spread), spread = the largest |z - max| with a weight that counts, at most 30 here."""
import gc
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
IGNORE = -100


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()                                 # (other modules count the device memory that is in use)


def grid(shape, dtype, seed, sigma, step, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.empty((shape[0], shape[1] + pad), device="cuda").normal_(0.0, sigma, generator=g)
    return (torch.round(t / step) * step).to(TORCH[dtype])[:, :shape[1]]


def operands(dtype, T, V, D, seed, pad=0, sigma=2.0, coarse=False):
    s = sigma / math.sqrt(D)
    step = 2.0 ** math.floor(math.log2(s)) / (1 if coarse else 32)
    return grid((T, D), dtype, seed, 1.0, 1.0 if coarse else 1 / 16, pad), grid((V, D), dtype, seed + 1, s, step, pad)


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def scores(gs, X, W, targets, top, scale=1.0, room=None, dtype=None):
    T, (V, D) = X.shape[0], W.shape
    dtype = dtype or {v: k for k, v in TORCH.items()}[X.dtype]
    out = {"logprob": torch.full((T,), 7.0, device="cuda"), "lse": torch.full((T,), 7.0, device="cuda"), "entropy": torch.full((T,), 7.0, device="cuda")}
    if top:
        out["top_index"] = torch.full((T, top), 7, dtype=torch.int64, device="cuda")
        out["top_logprob"] = torch.full((T, top), 7.0, device="cuda")
    n = gs.logprobs_workspace_bytes(dtype, T, V, D, top)
    gs.logprobs(X, W, targets=targets, scale=scale, ignore_index=IGNORE, workspace=workspace(n if room is None else room), **out)
    return out


def check(out, X, W, t, top, scale=1.0):
    z32 = (X.double() @ W.double().t()).float()                    # exact
    assert bool((z32.double() == X.double() @ W.double().t()).all())
    z32 = z32 * torch.tensor(scale, dtype=torch.float32, device="cuda") if scale != 1.0 else z32
    z = z32.double()
    lse = torch.logsumexp(z, 1)
    logs = z - lse[:, None]
    limit = 6e-6 + 4 * U * z.abs().amax(1) + 2 * U * lse.abs()
    assert bool(((out["lse"].double() - lse).abs() <= limit).all())
    entropy = torch.special.entr(logs.exp()).sum(1)
    assert bool(((out["entropy"].double() - entropy).abs() <= 8e-6 * 31).all()), float((out["entropy"].double() - entropy).abs().max())
    counts = t != IGNORE
    want = torch.where(counts, logs.gather(1, torch.where(counts, t, 0)[:, None])[:, 0], 0.0)
    assert bool(((out["logprob"].double() - want).abs() <= torch.where(counts, limit + 2 * U * want.abs(), 0.0)).all())
    if top:
        best = torch.sort(z32, dim=1, descending=True, stable=True)
        assert torch.equal(out["top_index"], best.indices[:, :top])
        want = best.values[:, :top].double() - lse[:, None]
        assert bool(((out["top_logprob"].double() - want).abs() <= limit[:, None] + 2 * U * want.abs()).all())


def targets_for(T, V, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    t[torch.rand(T, generator=g, device="cuda") < 0.2] = IGNORE
    t[0] = V - 1
    return t


SHAPES = [(1, 1, 1, 1), (1, 1000, 64, 5), (1, 50257, 128, 20), (2, 3, 5, 3), (3, 257, 40, 64), (7, 4099, 129, 8), (16, 5000, 768, 1), (33, 130, 64, 7), (64, 512, 256, 33),
          (129, 1003, 205, 20), (256, 4096, 128, 0), (500, 10007, 200, 8), (1027, 2048, 512, 64), (2048, 8192, 256, 5)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D,top", SHAPES)
def test_scores(gs, dtype, T, V, D, top):
    for pad, scale in ((0, 1.0), (3, 1 / 0.7)):
        X, W = operands(dtype, T, V, D, T + pad, pad)
        t = targets_for(T, V, T)
        check(scores(gs, X, W, t, top, scale), X, W, t, top, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,D,top", [(5, 700, 6, 17), (130, 3001, 4, 64), (64, 9000, 3, 8)])
def test_equal_logits_go_to_the_lowest_entry(gs, dtype, T, V, D, top):
    """A handful of different logits: nearly all are equal to many others, over tiles, sets and pieces."""
    X, W = operands(dtype, T, V, D, 3, coarse=True)
    t = targets_for(T, V, 3)
    check(scores(gs, X, W, t, top), X, W, t, top)
    X.zero_()                                                      # all of them
    out = scores(gs, X, W, t, top)
    assert torch.equal(out["top_index"], torch.arange(top, device="cuda").expand(T, top))
    assert bool(((out["entropy"].double() - math.log(V)).abs() <= 1e-5).all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
@pytest.mark.parametrize("order", ["drawn", "rising", "falling"])
def test_pieces_of_any_room(gs, dtype, order):
    """Less room, smaller pieces, the same entries: also where every piece's logits are larger, or smaller, than those before."""
    T, V, D, top = 70, 6001, 64, 12
    X, W = operands(dtype, T, V, D, 5)
    if order != "drawn":
        X = torch.ones_like(X)
        rank = torch.arange(V, device="cuda") if order == "rising" else torch.arange(V, device="cuda").flip(0)
        W = torch.zeros((V, D), device="cuda")
        W[:, 0], W[:, 1] = (rank // 64) / 16.0, (rank % 64) / 1024.0
        W = W.to(TORCH[dtype])
    t = targets_for(T, V, 5)
    full = gs.logprobs_workspace_bytes(dtype, T, V, D, top)
    tried = 0
    for part in (1.0, 0.5, 0.2, 0.1, 0.05):
        try:
            out = scores(gs, X, W, t, top, room=int(full * part) // 256 * 256)
        except gs.GensorError as e:
            assert e.status == 4
            continue
        check(out, X, W, t, top)
        tried += 1
    assert tried >= 3


@pytest.mark.parametrize("T,V,D,top", [(640, 120_000, 64, 8), (2100, 50257, 64, 16)])
def test_several_pieces_at_full_room(gs, T, V, D, top):
    X, W = operands("bf16", T, V, D, 9)
    t = targets_for(T, V, 9)
    check(scores(gs, X, W, t, top), X, W, t, top)


def test_targets_out_of_range_and_single_outputs(gs):
    X, W = operands("bf16", 6, 300, 64, 1)
    t = torch.tensor([0, 299, 300, -1, IGNORE, 2 ** 40], device="cuda")
    out = scores(gs, X, W, t, 3)
    assert torch.isfinite(out["logprob"][:2]).all() and torch.isnan(out["logprob"][[2, 3, 5]]).all() and float(out["logprob"][4]) == 0.0
    ws = workspace(gs.logprobs_workspace_bytes("bf16", 6, 300, 64, 3))
    for name in ("lse", "entropy"):
        one = torch.empty(6, device="cuda")
        gs.logprobs(X, W, workspace=ws, **{name: one})
        assert torch.equal(one, out[name])
    index, logprob = torch.empty((6, 3), dtype=torch.int64, device="cuda"), torch.empty((6, 3), device="cuda")
    gs.logprobs(X, W, top_index=index, top_logprob=logprob, workspace=ws)
    assert torch.equal(index, out["top_index"]) and torch.equal(logprob, out["top_logprob"])


def test_infinite_and_nan_logits(gs):
    """Entries that are shut off (minus infinity) are the last alternatives; a NaN is none; a token's own matter."""
    inf, nan = float("inf"), float("nan")
    X = torch.zeros((5, 4), device="cuda")
    X[:, 0] = 1.0
    W = torch.zeros((70, 4), device="cuda")
    W[:, 0] = -inf
    W[[3, 40, 41]] = torch.tensor([[1.0], [2.0], [2.0]], device="cuda").expand(3, 4) * torch.tensor([1.0, 0, 0, 0], device="cuda")
    t = torch.tensor([3, 40, 0, 41, IGNORE], device="cuda")
    out = scores(gs, X, W, t, 6)
    lse = math.log(math.e + 2 * math.e ** 2)
    assert out["top_index"].tolist() == [[40, 41, 3, 0, 1, 2]] * 5
    want = [2 - lse, 2 - lse, 1 - lse, -inf, -inf, -inf]
    assert all(a == b or abs(a - b) <= 4e-6 for a, b in zip(out["top_logprob"][2].tolist(), want))
    p = [math.exp(1 - lse), math.exp(2 - lse)]
    entropy = -p[0] * math.log(p[0]) - 2 * p[1] * math.log(p[1])
    assert bool(((out["entropy"] - entropy).abs() <= 1e-5).all())
    assert float(out["logprob"][2]) == -inf and abs(float(out["logprob"][1]) - (2 - lse)) <= 4e-6
    # NaN in one token's row only
    X[1, 0] = nan
    again = scores(gs, X, W, t, 6)
    keep = [0, 2, 3, 4]
    for k in out:
        assert torch.equal(again[k][keep], out[k][keep]), k
    assert math.isnan(float(again["lse"][1])) and math.isnan(float(again["entropy"][1])) and again["top_index"][1].tolist() == [-1] * 6
    assert bool(torch.isnan(again["top_logprob"][1]).all())
    # ... and in one entry: it is no alternative
    X[1, 0] = 1.0
    W[40, 0] = nan
    again = scores(gs, X, W, t, 6)
    assert again["top_index"].tolist() == [[41, 3, 0, 1, 2, 4]] * 5 and bool(torch.isnan(again["top_logprob"]).all())
    # infinite ones are alternatives in order, NaN none.  (The range overflows fp32: NaN, then inf up to the middle, -inf from there, and NaN)
    W[:, 0] = torch.linspace(-3e38, 3e38, 70)
    z = W[:, 0].cpu()
    assert bool(torch.isnan(z[[0, 69]]).all()) and bool((z[1:3] == inf).all())
    again = scores(gs, X, W, t, 2)
    assert again["top_index"].tolist() == [[1, 2]] * 5 and all(bool(torch.isnan(again[k]).all()) for k in ("lse", "entropy", "top_logprob"))
    # large logits: only differences count
    W[:, 0] = torch.linspace(-1, 1, 70, device="cuda") * 3e38
    again = scores(gs, X, W, t, 2)
    assert again["top_index"].tolist() == [[69, 68]] * 5 and float(again["top_logprob"][0, 0]) == 0.0 and bool((again["entropy"] == 0).all())


def test_a_token_alone_and_in_a_batch(gs):
    """Exact logits: the alternatives are the same, the sums within their rounding."""
    X, W = operands("bf16", 300, 5003, 128, 2)
    t = targets_for(300, 5003, 2)
    batch = scores(gs, X, W, t, 10)
    for i in (0, 151, 299):
        one = scores(gs, X[i:i + 1], W, t[i:i + 1], 10)
        assert torch.equal(one["top_index"][0], batch["top_index"][i])
        for k in ("logprob", "lse", "entropy", "top_logprob"):
            assert float((one[k][0] - batch[k][i]).abs().max()) <= 2e-5


def test_captured_and_replayed(gs):
    T, V, D, top = 90, 3000, 72, 9
    X, W = operands("f16", T, V, D, 6)
    t = targets_for(T, V, 6)
    ws = workspace(gs.logprobs_workspace_bytes("f16", T, V, D, top))
    out = {"logprob": torch.empty(T, device="cuda"), "entropy": torch.empty(T, device="cuda"), "top_index": torch.empty((T, top), dtype=torch.int64, device="cuda"),
           "top_logprob": torch.empty((T, top), device="cuda")}
    call = lambda: gs.logprobs(X, W, targets=t, workspace=ws, **out)
    call()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in out.items()}
    graph, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    for g in (graph, second):                                  # two graphs of one workspace
        with torch.cuda.graph(g):
            call()
    for n in range(3):
        for v in out.values():
            v.fill_(-5)
        ws.fill_(0xFF)                                         # (what is left there, NaN as numbers, does not count)
        (graph if n % 2 else second).replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for k in out), n
        X.neg_()
        second.replay()
        X.neg_()


def test_rows_far_apart(gs):
    """X the last token of long sequences: another tile, the room that was asked for."""
    T, V, D = 40, 2000, 256
    wide = torch.zeros((T, 6_000_000), device="cuda", dtype=torch.bfloat16)
    X, W = operands("bf16", T, V, D, 4)
    far = wide[:, -D:]
    far.copy_(X)
    t = targets_for(T, V, 4)
    check(scores(gs, far, W, t, 8), X, W, t, 8)


@pytest.mark.parametrize("T,V,D,top", [(1100, 3001, 4, 64), (1500, 30_000, 4, 9), (65, 20_000, 4, 33), (1025, 700, 3, 1)])
def test_equal_logits_of_many_tokens(gs, T, V, D, top):
    """More logits reach the bar than there is room for, with one wave a token and with several, in one piece and over many."""
    X, W = operands("bf16", T, V, D, 13, coarse=True)
    t = targets_for(T, V, 13)
    check(scores(gs, X, W, t, top), X, W, t, top)
    small = gs.logprobs_workspace_bytes("bf16", T, V, D, top) // 3 // 256 * 256
    check(scores(gs, X, W, t, top, room=small), X, W, t, top)
    X.zero_()
    assert torch.equal(scores(gs, X, W, t, top)["top_index"], torch.arange(top, device="cuda").expand(T, top))


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_operands_that_start_anywhere(gs, dtype):
    T, V, D, top = 37, 611, 64, 7
    X, W = operands(dtype, T, V, D, 21)
    t = targets_for(T, V, 21)
    want = scores(gs, X, W, t, top)
    for first, pad in ((1, 1), (3, 0), (1, 8)):
        def moved(m):
            flat = torch.full((m.shape[0] * (D + pad) + 8,), float("nan"), device="cuda").to(m.dtype)
            v = flat.as_strided(m.shape, (D + pad, 1), first)
            v.copy_(m)
            return v
        out = scores(gs, moved(X), moved(W), t, top)
        check(out, X, W, t, top)
        assert torch.equal(out["top_index"], want["top_index"])


def test_more_tokens_than_a_launch_has_workgroups_for(gs):
    T, V, D, top = 4_300_001, 5, 2, 2
    X, W = operands("f32", T, V, D, 17)
    t = targets_for(T, V, 17)
    check(scores(gs, X, W, t, top), X, W, t, top)


@pytest.mark.parametrize("T", [1, 256, 257, 1024, 1025])
def test_waves_a_token(gs, T):
    """On either side of the counts of tokens at which their number of waves changes, in one piece and in several."""
    V, D, top = 4001, 48, 11
    X, W = operands("f16", T, V, D, 23)
    t = targets_for(T, V, 23)
    n = gs.logprobs_workspace_bytes("f16", T, V, D, top)
    for room in (n, n // 4 // 256 * 256):
        check(scores(gs, X, W, t, top, room=room), X, W, t, top)


def test_sums_in_pieces_without_alternatives(gs):
    T, V, D = 300, 9001, 64
    X, W = operands("bf16", T, V, D, 27)
    t = targets_for(T, V, 27)
    n = gs.logprobs_workspace_bytes("bf16", T, V, D, 0)
    for part in (1.0, 0.5, 0.25):
        check(scores(gs, X, W, t, 0, 1 / 0.7, room=int(n * part) // 256 * 256), X, W, t, 0, 1 / 0.7)


@pytest.mark.parametrize("T", [3, 300, 1500])
@pytest.mark.parametrize("coarse", [False, True])
def test_larger_logits_in_later_pieces(gs, T, coarse):
    """Hundreds of a later piece's logits are above the largest so far, among them many equal ones."""
    V, D, top = 8003, 16, 9
    X, W = operands("bf16", T, V, D, 31, coarse=coarse)
    W[V // 4:] *= 4
    W[3 * V // 4:] *= 2
    t = targets_for(T, V, 31)
    n = gs.logprobs_workspace_bytes("bf16", T, V, D, top)
    for room in (n, n // 5 // 256 * 256, n // 12 // 256 * 256):
        check(scores(gs, X, W, t, top, room=room), X, W, t, top)


@pytest.mark.parametrize("T,V", [(1, 40_001), (6, 9001), (300, 9001), (1200, 40_001), (2200, 20_011)])
@pytest.mark.parametrize("top", [8, 25, 64])
@pytest.mark.parametrize("order", ["padded", "rising", "falling"])
def test_many_candidates(gs, T, V, top, order):
    """More logits than there is room for reach any bar that is known beforehand: a padded batch's tokens of zeros, whose logits are all equal, and
    logits in the order of their entries, with equal ones among them."""
    D = 16
    X, W = operands("bf16", T, V, D, 33)
    if order == "padded":
        X[T // 2:] = 0
    else:
        X = torch.ones_like(X)
        rank = torch.arange(V, device="cuda") if order == "rising" else torch.arange(V, device="cuda").flip(0)
        W = torch.zeros((V, D), device="cuda")
        W[:, 0], W[:, 1] = (rank // 512) / 16.0, (rank % 512 // 2) / 4096.0
        W = W.bfloat16()
    t = targets_for(T, V, 33)
    n = gs.logprobs_workspace_bytes("bf16", T, V, D, top)
    for room in (n, n // 7 // 256 * 256):
        check(scores(gs, X, W, t, top, room=room), X, W, t, top)


@pytest.mark.parametrize("T", [2, 1100])
def test_infinite_logits_among_many_equal(gs, T):
    """Hundreds of logits are plus infinity, or minus infinity, or NaN: the lowest of the equal entries, and -1 where no other is left."""
    V, D, top = 5003, 8, 40
    X, W = torch.zeros((T, D), device="cuda"), torch.zeros((V, D), device="cuda")
    X[:, 0] = 1.0
    W[1::2, 0] = math.inf
    for rest in (0.0, -math.inf, math.nan):
        W[0::2, 0] = rest
        out = scores(gs, X, W, targets_for(T, V, 5), top)
        assert torch.equal(out["top_index"], torch.arange(1, 2 * top, 2, device="cuda").expand(T, top))
    W.fill_(math.nan)
    W[7::1000] = 0.0
    W[7::1000, 0] = -math.inf
    out = scores(gs, X, W, targets_for(T, V, 5), top)
    want = torch.full((top,), -1, device="cuda")
    want[:5] = torch.arange(7, V, 1000, device="cuda")[:5]
    assert torch.equal(out["top_index"], want.expand(T, top))


def test_two_streams_at_once(gs):
    """Calls that overlap, each with a workspace of its own, give what they give alone."""
    shapes = [(700, 20_000, 128, 8), (3, 30_000, 64, 64), (1300, 6000, 96, 20)]
    calls, want = [], []
    for n, (T, V, D, top) in enumerate(shapes):
        X, W = operands("f16", T, V, D, 40 + n)
        t = targets_for(T, V, 40 + n)
        out = {"logprob": torch.empty(T, device="cuda"), "entropy": torch.empty(T, device="cuda"), "top_index": torch.empty((T, top), dtype=torch.int64, device="cuda"),
               "top_logprob": torch.empty((T, top), device="cuda")}
        ws = workspace(gs.logprobs_workspace_bytes("f16", T, V, D, top))
        calls.append((lambda X=X, W=W, t=t, ws=ws, out=out: gs.logprobs(X, W, targets=t, ignore_index=IGNORE, workspace=ws, **out), out, torch.cuda.Stream()))
        calls[-1][0]()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in out.items()})
    for _ in range(3):
        for call, out, stream in calls:
            for v in out.values():
                v.fill_(-5)
        torch.cuda.synchronize()
        for call, out, stream in calls:
            with torch.cuda.stream(stream):
                call()
                call()
        torch.cuda.synchronize()
        for (call, out, stream), w in zip(calls, want):
            assert all(torch.equal(out[k], w[k]) for k in out)
