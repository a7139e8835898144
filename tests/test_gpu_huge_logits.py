"""Logits of any finite size: a stretch of the vocabulary that is shut off by a large negative number, as long as a wave's rows or longer, and tokens all of whose
logits are huge, where only differences count.

Every logit is exact in fp32: a shut off one is -m itself (X's first column times W's, the others zero), a huge token's logits are
m times small whole numbers.  Tolerances, u = 2^-24: ordinary tokens as anywhere (6e-6 for exponentials, sums and joins, with 4 u |z| for the products, and 2 u |lse|
for lse's own rounding); those of huge tokens are single terms or equal ones: a term that is 1 may be a power of two times its inverse, each off by 2 u, and their product's rounding,
5 u together, and of equal ones' sums log's and lse's rounding are left."""
import gc
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FACTOR = 1.328125                                 # (a power of two times log2(e) needs no rounding)
SIZES = [FACTOR * 2.0 ** e for e in (20, 28, 29, 30, 31, 32, 33, 40, 60, 100, 121, 122, 126)]          # 1e6 to 1e38
NONE = -100


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()                                 # (other modules count the device memory that is in use)


def room(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def run(gs, dtype, X, W, t, top):
    """(lse, log probabilities, entropy, entries, their log probabilities) of the scores, and the loss and lse of the cross entropy and of a sure teacher."""
    T, (V, D) = X.shape[0], W.shape
    f = lambda *s: torch.full(s or (T,), 7.0, device="cuda")
    lse, logprob, entropy, index, values = f(), f(), f(), torch.full((T, top), 7, dtype=torch.int64, device="cuda"), f(T, top)
    gs.logprobs(X, W, targets=t, logprob=logprob, lse=lse, entropy=entropy, top_index=index, top_logprob=values, workspace=room(gs.logprobs_workspace_bytes(dtype, T, V, D, top)))
    loss, loss_lse, taught, taught_lse = f(), f(), f(), f()
    gs.xent_forward(X, W, t, loss, loss_lse, workspace=room(gs.xent_workspace_bytes(dtype, T, V, D)))
    gs.distill_forward(X, W, t[:, None].contiguous(), f(T, 1), taught, taught_lse, workspace=room(gs.distill_workspace_bytes(dtype, T, V, D, 1)))
    return lse, logprob, entropy, index, values, loss, loss_lse, taught, taught_lse


def far(m):
    """m as a product of two numbers of the type: the columns 0 of X and W."""
    e = int(math.log2(m))
    return 2.0 ** (e // 2), m / 2.0 ** (e // 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,D", [(1, 2000, 33), (70, 2000, 64), (300, 3001, 40), (2100, 1100, 64)])
def test_a_stretch_of_the_vocabulary_shut_off(gs, dtype, T, V, D):
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    x = torch.randint(-3, 4, (T, D), generator=g, device="cuda").float() / 8
    w = torch.randint(-3, 4, (V, D), generator=g, device="cuda").float() / 4
    off = torch.zeros(V, dtype=torch.bool, device="cuda")
    off[300:900] = True                                              # whole tiles
    off[V - 130:] = True                                             # and the end, as a vocabulary is padded
    w[off] = 0
    z = (x[:, 1:].double() @ w[:, 1:].double().t())[:, ~off]
    entries = torch.arange(V, device="cuda")[~off]
    t = entries[torch.randint(0, len(entries), (T,), generator=g, device="cuda")]
    lse = torch.logsumexp(z, 1)
    logs = z - lse[:, None]
    best = torch.sort(z, dim=1, descending=True, stable=True)
    at = logs.gather(1, torch.searchsorted(entries, t)[:, None])[:, 0]
    entropy = torch.special.entr(logs.exp()).sum(1)
    limit = 6e-6 + 4 * U * z.abs().amax(1) + 2 * U * lse.abs()
    for m in SIZES:
        a, b = far(m)
        x[:, 0] = a
        w[:, 0] = torch.where(off, -b, 0.0)
        X, W = x.to(TORCH[dtype]), w.to(TORCH[dtype])
        got = run(gs, dtype, X, W, t, 5)
        for i in (0, 6, 8):
            assert bool(((got[i].double() - lse).abs() <= limit).all()), (m, i, float((got[i].double() - lse).abs().max()))
        for i, sign in ((1, 1), (5, -1), (7, -1)):
            assert bool(((sign * got[i].double() - at).abs() <= limit + 2 * U * at.abs()).all()), (m, i)
        assert bool(((got[2].double() - entropy).abs() <= 8e-6 * (1 + float((z.amax(1) - z.amin(1)).max()))).all()), m
        assert torch.equal(got[3], entries[best.indices[:, :5]]), m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(3, 700), (80, 2000), (1100, 600)])
def test_tokens_of_huge_logits(gs, dtype, T, V):
    """m times 1 for one entry and 0 or -1 for the others, all of them -m, and m: alone and beside ordinary tokens."""
    D = 16
    t = torch.full((T,), V // 2, device="cuda")
    for m in SIZES:
        a, b = far(m)
        W = torch.zeros((V, D), device="cuda")
        W[:, 0] = -(torch.arange(V, device="cuda") % 2) * b
        W[V // 2, 0], W[:, 1], W[:, 2] = b, -b, b
        X = torch.zeros((T, D), device="cuda")
        X[0::3, 0], X[1::3, 1], X[2::3, 2] = a, a, a
        X[0] = 0                                                     # (an ordinary token: all logits are zero)
        got = run(gs, dtype, X.to(TORCH[dtype]), W.to(TORCH[dtype]), t, 4)
        kind = torch.arange(T, device="cuda") % 3
        log_v = math.log(V)
        one, low, high = (kind == 0), (kind == 1), (kind == 2)
        one[0] = False
        for i, want in ((0, m), (1, 0.0), (2, 0.0), (5, 0.0), (6, m), (7, 0.0), (8, m)):
            assert bool(((got[i][one] - want).abs() <= 5 * U).all()), (m, i)         # the others' exponentials vanish
        assert bool((got[3][one][:, 0] == V // 2).all()) and bool((got[4][one][:, 0] == 0).all())
        for which, size in ((low, -m), (high, m)):
            for i in (0, 6, 8):
                assert bool(((got[i][which].double() - (size + log_v)).abs() <= U * m + 4 * U * log_v).all()), (m, i)
            for i, want in ((1, -log_v), (2, log_v)):
                assert bool(((got[i][which].double() - want).abs() <= 2e-6).all()), (m, i)
            assert bool((got[3][which] == torch.arange(4, device="cuda")).all()), m
            assert bool(((got[4][which].double() + log_v).abs() <= 2e-6).all()), m
        assert abs(float(got[0][0]) - log_v) <= 2e-6 and abs(float(got[6][0]) - log_v) <= 2e-6 and abs(float(got[8][0]) - log_v) <= 2e-6
