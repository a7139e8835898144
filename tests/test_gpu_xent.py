"""Cross entropy of a projection (logits never stored) and its gradient against the definition in 64 bits.

Tolerances.  u = 2^-24.  A logit is off by at most e_z = (D + 1) u sum|x||w|; lse moves by no more than its largest logit error, and by the
rounding of the exponentials' arguments and sums, at most 2e-6 + u |lse| here (exponents below 30, slabs and joins of a few thousand terms);
loss by both.  A probability is then off by a factor 1 + 2 e_z + 4e-6 + u |lse|; G is rounded to the type (f16: after scaling, whose
subnormal step is 2^-39 of the largest |dloss|); a product's sums of n terms are off by (n + 1) u sum|G||w|; results are rounded once."""
import gc
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}
IGNORE = -100


@pytest.fixture(scope="module")
def gs():
    from paper_2502_11407_amd import binding
    yield binding
    gc.collect()                                 # (other modules count the device memory that is in use)


def draw(shape, dtype, seed, sigma=1.0, pad=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty((shape[0], shape[1] + pad), device="cuda").normal_(0.0, sigma, generator=g).to(TORCH[dtype])[:, :shape[1]]


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


def inputs(dtype, T, V, D, pad, seed, ignored=0.2, sigma=2.0):
    X, W = draw((T, D), dtype, seed, 1.0, pad), draw((V, D), dtype, seed + 1, sigma / math.sqrt(D), pad)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 2)
    t = torch.randint(0, V, (T,), generator=g, device="cuda")
    t[torch.rand(T, generator=g, device="cuda") < ignored] = IGNORE
    t[0] = V - 1
    return X, W, t


def reference(X, W, t):
    x, w = X.double(), W.double()
    z = x @ w.t()
    lse = torch.logsumexp(z, 1)
    counts = t != IGNORE
    at = torch.where(counts, t, torch.zeros_like(t))
    loss = torch.where(counts, lse - z.gather(1, at[:, None])[:, 0], torch.zeros_like(lse))
    e_z = (x.shape[1] + 1) * U * (x.abs() @ w.abs().t()).amax(1)
    return z, lse, loss, counts, at, e_z


def check_gradient(dtype, X, W, t, lse, dloss, dX, dW):
    z, lse64, _, counts, at, e_z = reference(X, W, t)
    x, w = X.double(), W.double()
    p = torch.exp(z - lse.double()[:, None])
    g = torch.where(counts, dloss.double(), torch.zeros_like(lse64))[:, None]
    one = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    G = (p - one) * g
    top = float(dloss.abs().max())
    step = top * 2.0 ** -39 if dtype == "f16" else 0.0
    e_g = (ROUND[dtype] * 1.01 + 2 * U) * G.abs() + p * g.abs() * (2 * e_z[:, None] + 4e-6 + 2 * U * lse64.abs()[:, None]) + 2 * U * g.abs() * one + step
    for got, want, bound in ((dX, G @ w, e_g @ w.abs() + (W.shape[0] + 8) * U * (G.abs() @ w.abs())),
                             (dW, G.t() @ x, e_g.t() @ x.abs() + (X.shape[0] + 8) * U * (G.abs().t() @ x.abs()))):
        if got is None:
            continue
        limit = 1.01 * bound + ROUND[dtype] * want.abs() + TINY[dtype]
        bad = ~((got.double() - want).abs() <= limit)
        assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - want).abs() / limit).nan_to_num(1e9).max()), torch.nonzero(bad)[:3].tolist())


SHAPES = [(1, 1, 1), (1, 1000, 64), (2, 3, 5), (3, 257, 40), (7, 4099, 129), (16, 5000, 768), (33, 130, 64), (64, 512, 256), (129, 1003, 205),
          (256, 4096, 128), (500, 10007, 200), (1027, 2048, 512), (2048, 8192, 256)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D", SHAPES)
def test_loss_and_gradient(gs, dtype, T, V, D):
    for pad in (0, 3):
        X, W, t = inputs(dtype, T, V, D, pad, T + V)
        loss, lse = torch.full((T + 1,), 7.0, device="cuda"), torch.full((T + 1,), 7.0, device="cuda")
        gs.xent_forward(X, W, t, loss[:T], lse[:T], ignore_index=IGNORE, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D)))
        _, lse64, loss64, counts, _, e_z = reference(X, W, t)
        limit = e_z + 2e-6 + 2 * U * lse64.abs()
        assert bool(((lse[:T].double() - lse64).abs() <= limit).all()), float(((lse[:T].double() - lse64).abs() / limit).max())
        assert bool(((loss[:T].double() - loss64).abs() <= 2 * limit).all())
        assert bool((loss[:T][~counts] == 0).all()) and float(loss[T]) == 7.0 and float(lse[T]) == 7.0
        dloss = draw((1, T), "f32", 9)[0].contiguous() * (1.0 / T)
        dX = torch.full((T + 1, D + pad), 7.0, dtype=TORCH[dtype], device="cuda")
        dW = torch.full((V + 1, D + pad), 7.0, dtype=TORCH[dtype], device="cuda")
        gs.xent_backward(X, W, t, lse[:T], dloss, dX[:T, :D], dW[:V, :D], ignore_index=IGNORE,
                         workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D, backward=True)))
        check_gradient(dtype, X, W, t, lse[:T], dloss, dX[:T, :D], dW[:V, :D])
        for m, n in ((dX, T), (dW, V)):
            assert bool((m[n] == 7).all()) and bool((m[:, D:] == 7).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T", [40, 77])
def test_pieces(gs, dtype, T):
    """A workspace of less than is asked for: more, smaller pieces of the vocabulary, the same gradient; too little is refused."""
    V, D = 2500, 96
    X, W, t = inputs(dtype, T, V, D, 0, 5)
    lse = torch.empty(T, device="cuda")
    gs.xent_forward(X, W, t, None, lse, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D)))
    dloss = torch.full((T,), 1.0 / T, device="cuda")
    need, es = gs.xent_workspace_bytes(dtype, T, V, D, backward=True), 4 if dtype == "f32" else 2
    pitch = (T + 7) // 8 * 8
    least = 256 + pitch * D * es + T * D * 4 + 256 * pitch * es + 1024
    for room in (need, least + 700 * pitch * es, least):
        dX, dW = torch.empty((T, D), dtype=TORCH[dtype], device="cuda"), torch.empty((V, D), dtype=TORCH[dtype], device="cuda")
        gs.xent_backward(X, W, t, lse, dloss, dX, dW, workspace=workspace(room))
        check_gradient(dtype, X, W, t, lse, dloss, dX, dW)
    with pytest.raises(gs.GensorError, match="WORKSPACE"):
        gs.xent_backward(X, W, t, lse, dloss, dX, dW, workspace=workspace(256 * pitch * es))
    with pytest.raises(gs.GensorError, match="WORKSPACE"):
        gs.xent_forward(X, W, t, None, lse, workspace=workspace(256))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128, 192, 256, 328, 768])
def test_more_tiles_than_compute_units(gs, dtype, D):
    """Workgroups that take several tiles of the logits: one to many k tiles, the last tiles ragged in both directions."""
    T, V = 2310, 9000
    X, W, t = inputs(dtype, T, V, D, 0, D)
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    gs.xent_forward(X, W, t, loss, lse, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D)))
    _, lse64, loss64, _, _, e_z = reference(X, W, t)
    limit = e_z + 2e-6 + 2 * U * lse64.abs()
    assert bool(((lse.double() - lse64).abs() <= limit).all()), float(((lse.double() - lse64).abs() / limit).max())
    assert bool(((loss.double() - loss64).abs() <= 2 * limit).all())


def test_one_gradient_of_the_two(gs):
    T, V, D = 100, 1500, 128
    X, W, t = inputs("bf16", T, V, D, 0, 5)
    lse, dloss = torch.empty(T, device="cuda"), torch.full((T,), 0.01, device="cuda")
    ws = workspace(gs.xent_workspace_bytes("bf16", T, V, D, backward=True))
    gs.xent_forward(X, W, None, None, lse, workspace=workspace(gs.xent_workspace_bytes("bf16", T, V, D)))
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    gs.xent_backward(X, W, t, lse, dloss, dX, None, workspace=ws)
    gs.xent_backward(X, W, t, lse, dloss, None, dW, workspace=ws)
    check_gradient("bf16", X, W, t, lse, dloss, dX, dW)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_all_ignored_and_targets_outside(gs, dtype):
    T, V, D = 20, 300, 64
    X, W, t = inputs(dtype, T, V, D, 0, 5)
    for values, want in ((IGNORE, 0.0), (V, math.nan), (-1, math.nan), (2 ** 40, math.nan)):
        t.fill_(values)
        loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        gs.xent_forward(X, W, t, loss, lse, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D)))
        assert bool((loss == 0).all()) if want == 0.0 else bool(torch.isnan(loss).all())
        dX, dW = torch.full_like(X, 5.0), torch.full_like(W, 5.0)
        gs.xent_backward(X, W, t, lse, torch.ones(T, device="cuda"), dX, dW, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D, backward=True)))
        assert bool((dX == 0).all()) and bool((dW == 0).all())


def test_confident_and_extreme_logits(gs):
    """A token that its target dominates loses log(1 + the rest), not a rounding; infinite logits give infinite or undefined losses as the
    definition does, and leave other tokens alone."""
    T, V, D = 4, 700, 8
    X, W = torch.zeros((T, D), device="cuda"), torch.zeros((V, D), device="cuda")
    X[:, 0] = 1.0
    W[5, 0] = 30.0
    W[:, 1] = 1.0
    X[1, 0], X[1, 1] = 0.0, math.inf                        # every logit of token 1 is infinite (0 * 30 beside it)
    X[2, 0], X[2, 1] = 0.0, -3e38                           # the type's lowest values
    t = torch.full((T,), 5, device="cuda")
    t[3] = 6
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    gs.xent_forward(X, W, t, loss, lse, workspace=workspace(gs.xent_workspace_bytes("f32", T, V, D)))
    rest = 699 * math.exp(-30)
    assert abs(float(loss[0]) - rest) <= 1e-3 * rest + 2 * U and float(loss[0]) >= 0
    assert float(lse[1]) == math.inf and math.isnan(float(loss[1]))
    assert abs(float(lse[2]) + 3e38) < 1e32 and abs(float(loss[2]) - math.log(700)) < 1e-4
    assert abs(float(loss[3]) - 30) < 1e-4


def test_gradient_against_differences(gs):
    """d loss / d x by central differences of the forward, in fp32."""
    T, V, D = 6, 50, 12
    X, W, t = inputs("f32", T, V, D, 0, 11, ignored=0.0)
    ws, h = workspace(gs.xent_workspace_bytes("f32", T, V, D)), 2.0 ** -6
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")

    def value(x, w):
        gs.xent_forward(x, w, t, loss, lse, workspace=ws)
        return loss.double()

    value(X, W)
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    gs.xent_backward(X, W, t, lse.clone(), torch.ones(T, device="cuda"), dX, dW, workspace=workspace(gs.xent_workspace_bytes("f32", T, V, D, backward=True)))
    # error: h^2 / 6 times the third derivative along one coordinate (at most max|w|^3), and 2 * 4e-6 / (2 h) of rounding
    for d in range(D):
        step = torch.zeros_like(X)
        step[:, d] = h
        slope = (value(X + step, W) - value(X - step, W)) / (2 * h)
        assert float((slope - dX[:, d].double()).abs().max()) <= h * h / 6 * float(W.abs().max()) ** 3 + 4e-6 / h + 1e-5
    for v, d in ((0, 0), (7, 3), (49, 11), (int(t[0]), 5)):
        step = torch.zeros_like(W)
        step[v, d] = h
        slope = ((value(X, W + step) - value(X, W - step)) / (2 * h)).sum()
        assert abs(float(slope - dW[v, d].double())) <= T * (h * h / 6 * float(X.abs().max()) ** 3 + 4e-6 / h + 1e-5)


def test_f16_gradients_of_a_mean_keep_their_digits(gs):
    """dloss far below f16's normal range: scaled inside, so that dX (made of ordinary weights) keeps f16's precision."""
    T, V, D = 64, 3000, 64
    X, W, t = inputs("f16", T, V, D, 0, 3)
    lse = torch.empty(T, device="cuda")
    gs.xent_forward(X, W, t, None, lse, workspace=workspace(gs.xent_workspace_bytes("f16", T, V, D)))
    for top in (1e-7, 1.0, 3e4):
        dloss = torch.linspace(0.1, 1.0, T, device="cuda") * top
        dX, dW = torch.empty_like(X), torch.empty_like(W)
        gs.xent_backward(X, W, t, lse, dloss, dX, dW, workspace=workspace(gs.xent_workspace_bytes("f16", T, V, D, backward=True)))
        if top < 3e4:                        # (results beyond f16's largest value are infinite)
            check_gradient("f16", X, W, t, lse, dloss, dX, dW)
    zero = torch.zeros(T, device="cuda")
    gs.xent_backward(X, W, t, lse, zero, dX, dW, workspace=workspace(gs.xent_workspace_bytes("f16", T, V, D, backward=True)))
    assert bool((dX == 0).all()) and bool((dW == 0).all())


def test_graph_replays(gs):
    T, V, D = 200, 3000, 128
    X, W, t = inputs("f16", T, V, D, 0, 3)
    loss, lse, dloss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.full((T,), 1.0 / T, device="cuda")
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    ws, bws = workspace(gs.xent_workspace_bytes("f16", T, V, D)), workspace(gs.xent_workspace_bytes("f16", T, V, D, backward=True))

    def step():
        gs.xent_forward(X, W, t, loss, lse, workspace=ws)
        gs.xent_backward(X, W, t, lse, dloss, dX, dW, workspace=bws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (7, 8, 9):
        X.copy_(draw((T, D), "f16", seed))
        graph.replay()
        torch.cuda.synchronize()
        got = [v.clone() for v in (loss, lse, dX, dW)]
        step()
        for a, b in zip(got, (loss, lse, dX, dW)):
            assert torch.equal(a, b)
