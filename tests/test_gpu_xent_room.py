"""The loss with any room: what gensor_xent_workspace_bytes asks for serves rows at any distance, and less takes the vocabulary in pieces."""
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


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def check(gs, dtype, X, W, t, ws):
    """Both results against 64 bits: a logit is off by at most (D + 1) u sum|x||w|, lse by the largest of them and 2e-6 + 2 u |lse| of the
    exponentials and sums, the loss by twice that."""
    T = X.shape[0]
    loss, lse = torch.full((T + 1,), 7.0, device="cuda"), torch.full((T + 1,), 7.0, device="cuda")
    gs.xent_forward(X, W, t, loss[:T], lse[:T], ignore_index=IGNORE, workspace=ws)
    x, w = X.double(), W.double()
    z = x @ w.t()
    lse64 = torch.logsumexp(z, 1)
    counts = t != IGNORE
    loss64 = torch.where(counts, lse64 - z.gather(1, torch.where(counts, t, torch.zeros_like(t))[:, None])[:, 0], torch.zeros_like(lse64))
    limit = (x.shape[1] + 1) * U * (x.abs() @ w.abs().t()).amax(1) + 2e-6 + 2 * U * lse64.abs()
    assert bool(((lse[:T].double() - lse64).abs() <= limit).all()), float(((lse[:T].double() - lse64).abs() / limit).max())
    assert bool(((loss[:T].double() - loss64).abs() <= 2 * limit).all()), float(((loss[:T].double() - loss64).abs() / limit).max())
    assert bool((loss[:T][~counts] == 0).all()) and float(loss[T]) == 7.0 and float(lse[T]) == 7.0
    return loss[:T].clone(), lse[:T].clone()


def targets(T, V, seed):
    """Targets all over the vocabulary, its first and last entries among them, and some that are ignored."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    t[torch.rand(T, generator=g, device="cuda") < 0.1] = IGNORE
    t[0], t[T - 1] = V - 1, 0
    return t


@pytest.mark.parametrize("dtype,T,V,D,S", [("bf16", 128, 50257, 4096, 2048), ("f16", 64, 32000, 4096, 4096), ("bf16", 512, 50257, 1024, 8192), ("f32", 64, 5003, 1024, 8192)])
def test_last_token_of_each_sequence(gs, dtype, T, V, D, S):
    """X = hidden[:, -1, :]: its rows are S * D apart, further than large tiles reach.  The asked-for workspace serves as it does for rows side by side."""
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    X = torch.empty((T, S, D), dtype=TORCH[dtype], device="cuda")[:, -1, :]
    X.copy_(torch.empty((T, D), device="cuda").normal_(0.0, 1.0, generator=g))
    W = torch.empty((V, D), device="cuda").normal_(0.0, 2.0 / math.sqrt(D), generator=g).to(TORCH[dtype])
    check(gs, dtype, X, W, targets(T, V, 1), workspace(gs.xent_workspace_bytes(dtype, T, V, D)))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D", [(1, 1000, 64), (5, 2500, 96), (77, 4099, 41), (300, 5000, 128), (2310, 9000, 128)])
def test_less_room(gs, dtype, T, V, D):
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    X = torch.empty((T, D), device="cuda").normal_(0.0, 1.0, generator=g).to(TORCH[dtype])
    W = torch.empty((V, D), device="cuda").normal_(0.0, 2.0 / math.sqrt(D), generator=g).to(TORCH[dtype])
    t, need, head = targets(T, V, 2), gs.xent_workspace_bytes(dtype, T, V, D), (4 * T + 255) // 256 * 256
    check(gs, dtype, X, W, t, workspace(need))
    # (the least: what pieces have joined to, and the slabs of a row of tiles, at most four)
    least = head + 2 * ((5 * 4 * T + 255) // 256 * 256)
    for room in (max(need - 1, least), (need + least) // 2, least + (need - least) // 7, least):
        got = check(gs, dtype, X, W, t, workspace(room))
        again = check(gs, dtype, X, W, t, workspace(room))
        assert all(torch.equal(a, b) for a, b in zip(got, again))
    lse = torch.empty(T, device="cuda")
    gs.xent_forward(X, W, None, None, lse, workspace=workspace(least))
    assert torch.equal(lse, got[1])
    with pytest.raises(gs.GensorError, match="WORKSPACE"):
        gs.xent_forward(X, W, t, None, lse, workspace=workspace(head))


def test_pieces_without_a_finite_logit(gs):
    """A piece whose every logit is -inf leaves what the others have; an infinite logit in one piece decides."""
    V = 3000
    X, W = torch.ones((1, 1), device="cuda"), torch.full((V, 1), -math.inf, device="cuda")
    W[17, 0], W[2999, 0] = 1.5, 2.5
    ws = workspace(256 + 2 * 256)                # (sums of 63 slabs at most in a piece)
    loss, lse = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    t = torch.tensor([17], device="cuda")
    gs.xent_forward(X, W, t, loss, lse, workspace=ws)
    want = 2.5 + math.log(1 + math.exp(-1.0))
    assert abs(float(lse[0]) - want) < 1e-5 and abs(float(loss[0]) - (want - 1.5)) < 1e-5
    W[1500, 0] = math.inf
    gs.xent_forward(X, W, t, loss, lse, workspace=ws)
    assert float(lse[0]) == math.inf and float(loss[0]) == math.inf


def test_graph_of_pieces(gs):
    T, V, D = 200, 6000, 128
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    X = torch.empty((T, D), device="cuda").normal_(0.0, 1.0, generator=g).to(torch.bfloat16)
    W = torch.empty((V, D), device="cuda").normal_(0.0, 0.2, generator=g).to(torch.bfloat16)
    t, ws = targets(T, V, 3), workspace(1024 + 2 * 8192)
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")

    def step():
        gs.xent_forward(X, W, t, loss, lse, ignore_index=IGNORE, workspace=ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        X.copy_(torch.empty((T, D), device="cuda").normal_(0.0, 1.0, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        got = loss.clone(), lse.clone()
        step()
        assert torch.equal(got[0], loss) and torch.equal(got[1], lse)
