"""The distillation loss against a teacher's top entries and its gradient (logits never stored) against the definition in 64 bits.

Tolerances.  u = 2^-24.  A logit is off by at most e_z = (D + 2) u scale sum|x||w|; lse moves by no more than its largest logit error and by the rounding of
exponentials, sums and joins, 4e-6 + 2 u |lse| here; a teacher's p by a factor 1 + 4e-6 + 4 u |log p| (the exponential, the sum over the
entries); the loss by P (e_z + that of lse) + sum p (4e-6 + ...) (1 + |log p - z + lse|).  A probability is off by a factor 1 + 2 e_z + 4e-6 + 2 u |lse|; G
is rounded to the type (f16: after scaling, whose subnormal step is 2^-39 of the largest weight); a product's sum of n terms is off by
(n + 8) u sum|G||w|; results are rounded once."""
import gc
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ROUND = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}


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
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def inputs(dtype, T, V, D, k, pad, seed):
    """Some entries twice, some tokens with fewer entries (holes among them) and some with none; what stands at a hole is no number."""
    X, W = draw((T, D), dtype, seed, 1.0, pad), draw((V, D), dtype, seed + 1, 2 / math.sqrt(D), pad)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 2)
    index = torch.randint(0, V, (T, k), generator=g, device="cuda")
    q = -3 * torch.rand((T, k), generator=g, device="cuda") - 0.5 - math.log(k)
    q[:, -1] = -float("inf") if k > 2 else q[:, -1]
    hole = torch.rand((T, k), generator=g, device="cuda") < 0.2
    hole |= (torch.rand(T, generator=g, device="cuda") < 0.1)[:, None]
    index, q = torch.where(hole, -1, index), torch.where(hole, float("nan"), q)
    index[0, 0], q[0, 0] = V - 1, -0.25
    if k > 1:
        index[0, 1], q[0, 1] = V - 1, -1.0                         # the same entry twice
    return X, W, index.contiguous(), q.contiguous()


def probabilities(index, q, scale, normalize):
    q = torch.where(index >= 0, q.double(), -float("inf"))
    if normalize:
        q = scale * q
        some = torch.isfinite(q).any(1, keepdim=True)
        q = torch.where(some, q - torch.logsumexp(torch.where(some, q, 0.0), 1, keepdim=True), -float("inf"))
    return torch.exp(q), q


def reference(X, W, index, q, scale, normalize):
    x, w = X.double(), W.double()
    z = scale * (x @ w.t())
    lse = torch.logsumexp(z, 1)
    p, logp = probabilities(index, q, scale, normalize)
    each = torch.where(p > 0, logp - z.gather(1, index.clamp(min=0)) + lse[:, None], 0.0)
    e_z = scale * (x.shape[1] + 2) * U * (x.abs() @ w.abs().t()).amax(1)
    return z, lse, p, torch.where(p > 0, logp, 0.0), each, e_z


def check_forward(loss, lse, ref):
    z, lse64, p, logp, each, e_z = ref
    e_lse = e_z + 4e-6 + 2 * U * lse64.abs()
    assert bool(((lse.double() - lse64).abs() <= 1.01 * e_lse).all())
    bound = (p * (e_z + e_lse)[:, None]).sum(1) + (p * (6e-6 + 8 * U * logp.abs() + (len(p[0]) + 8) * U) * (1 + each.abs())).sum(1)
    off = (loss.double() - (p * each).sum(1)).abs()
    assert bool((off <= 1.01 * bound).all()), float((off / bound).nan_to_num(0).max())


def check_gradient(dtype, X, W, index, q, scale, normalize, lse, dloss, dX, dW):
    z, lse64, p, logp, _, e_z = reference(X, W, index, q, scale, normalize)
    x, w = X.double(), W.double()
    s = torch.exp(z - lse.double()[:, None])
    mass = p.sum(1, keepdim=True)
    hot = torch.zeros_like(s).scatter_add_(1, index.clamp(min=0), p)
    g = scale * dloss.double()[:, None]
    G = (mass * s - hot) * g
    step = float((g * mass).abs().max()) * 2.0 ** -39 if dtype == "f16" else 0.0
    e_p = 6e-6 + 8 * U * logp.abs().amax(1, keepdim=True) + (p.shape[1] + 8) * U
    e_g = ((ROUND[dtype] * 1.01 + 4 * U) * G.abs() + mass * s * g.abs() * (2 * e_z[:, None] + 4e-6 + 2 * U * lse64.abs()[:, None] + e_p) + hot * g.abs() * e_p + step)
    for got, want, bound in ((dX, G @ w, e_g @ w.abs() + (W.shape[0] + 8) * U * (G.abs() @ w.abs())),
                             (dW, G.t() @ x, e_g.t() @ x.abs() + (X.shape[0] + 8) * U * (G.abs().t() @ x.abs()))):
        if got is None:
            continue
        limit = 1.01 * bound + ROUND[dtype] * want.abs() + TINY[dtype]
        bad = ~((got.double() - want).abs() <= limit)
        assert not bool(bad.any()), (int(bad.sum()), float(((got.double() - want).abs() / limit).nan_to_num(1e9).max()), torch.nonzero(bad)[:3].tolist())


def forward(gs, X, W, index, q, scale=1.0, normalize=True):
    dtype = {v: k for k, v in TORCH.items()}[X.dtype]
    T, (V, D), k = X.shape[0], W.shape, index.shape[1]
    loss, lse = torch.full((T,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
    gs.distill_forward(X, W, index, q, loss, lse, scale=scale, normalize=normalize, workspace=workspace(gs.distill_workspace_bytes(dtype, T, V, D, k)))
    return loss, lse


def backward(gs, X, W, index, q, lse, dloss, scale=1.0, normalize=True, room=None, want=(True, True)):
    dtype = {v: k for k, v in TORCH.items()}[X.dtype]
    T, (V, D), k = X.shape[0], W.shape, index.shape[1]
    dX, dW = (torch.full(s, 7.0, device="cuda").to(X.dtype) if yes else None for s, yes in zip(((T, D), (V, D)), want))
    n = gs.distill_workspace_bytes(dtype, T, V, D, k, backward=True) if room is None else room
    gs.distill_backward(X, W, index, q, lse, dloss, dX, dW, scale=scale, normalize=normalize, workspace=workspace(n))
    return dX, dW


SHAPES = [(1, 1, 1, 1), (1, 1000, 64, 5), (2, 3, 5, 3), (3, 257, 40, 64), (7, 4099, 129, 8), (16, 5000, 768, 1), (33, 130, 64, 256), (64, 512, 256, 33), (129, 1003, 205, 20),
          (256, 4096, 128, 4), (500, 10007, 200, 16), (1027, 2048, 512, 64)]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("T,V,D,k", SHAPES)
def test_loss_and_gradient(gs, dtype, T, V, D, k):
    for pad, scale, normalize in ((0, 1.0, True), (3, 0.5, False), (0, 1 / 0.7, True)):
        X, W, index, q = inputs(dtype, T, V, D, k, pad, T + k)
        loss, lse = forward(gs, X, W, index, q, scale, normalize)
        check_forward(loss, lse, reference(X, W, index, q, scale, normalize))
        empty = ~(index >= 0).any(1)
        assert bool((loss[empty] == 0).all())
        g = torch.Generator(device="cuda")
        g.manual_seed(T)
        dloss = (torch.rand(T, generator=g, device="cuda") - 0.3) * (64.0 if dtype == "f16" else 1.0) / T
        dX, dW = backward(gs, X, W, index, q, lse, dloss, scale, normalize)
        check_gradient(dtype, X, W, index, q, scale, normalize, lse, dloss, dX, dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_entry_is_cross_entropy(gs, dtype):
    """A teacher that is sure: the loss and the gradient of xent_forward and xent_backward, within the rounding of either's sums."""
    T, V, D = 150, 3001, 96
    X, W = draw((T, D), dtype, 1), draw((V, D), dtype, 2, 0.2)
    t = torch.randint(0, V, (T,), generator=torch.Generator("cuda").manual_seed(3), device="cuda")
    loss, lse = forward(gs, X, W, t[:, None].contiguous(), torch.full((T, 1), -3.0, device="cuda"))
    plain, plain_lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    gs.xent_forward(X, W, t, plain, plain_lse, workspace=workspace(gs.xent_workspace_bytes(dtype, T, V, D)))
    assert float((loss - plain).abs().max()) <= 2e-5 and float((lse - plain_lse).abs().max()) <= 1e-5
    dloss = torch.full((T,), 1.0 / T, device="cuda")
    dX, dW = backward(gs, X, W, t[:, None].contiguous(), torch.full((T, 1), -3.0, device="cuda"), lse, dloss)
    check_gradient(dtype, X, W, t[:, None], torch.full((T, 1), -3.0, device="cuda"), 1.0, True, lse, dloss, dX, dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_against_differences(gs, dtype):
    """The gradient of the loss itself along a drawn direction, by central differences of the forward.  The step's own curvature, h^2 / 6 times the third derivative (below 4
    |direction's logits|^3, these below 0.2), and 4e-6 losses' rounding over h."""
    T, V, D, k = 24, 400, 48, 6
    X, W, index, q = inputs("f32", T, V, D, k, 0, 11)
    loss, lse = forward(gs, X, W, index, q)
    dloss = torch.linspace(0.5, 1.5, T, device="cuda")
    if dtype != "f32":
        X, W = X.to(TORCH[dtype]), W.to(TORCH[dtype])
        loss, lse = forward(gs, X, W, index, q)
    dX, dW = backward(gs, X, W, index, q, lse, dloss)
    x, w, h = X.float(), W.float(), 2.0 ** -4
    for direction, grad, move in ((draw((T, D), "f32", 12, 0.02), dX, lambda d: (x + d, w)), (draw((V, D), "f32", 13, 0.02), dW, lambda d: (x, w + d))):
        up, down = (forward(gs, *move(s * h * direction), index, q)[0] for s in (1.0, -1.0))
        slope = ((up - down).double() * dloss).sum() / (2 * h)
        got = (grad.double() * direction.double()).sum()
        third = T * 1.5 * 4 * 0.2 ** 3 * h * h / 6
        noise = 2 * 4e-6 * float(dloss.sum()) * 8 / (2 * h)
        rounding = 2.5 * ROUND[dtype] * float((grad.double().abs() * direction.double().abs()).sum())      # G's and the result's
        assert abs(float(slope - got)) <= third + noise + rounding


def test_tokens_that_teach_nothing(gs):
    """No entries, probabilities of zero, a gradient of zero, entries out of range: no gradient, whatever their rows of logits are."""
    T, V, D, k = 12, 600, 64, 4
    X, W, index, q = inputs("bf16", T, V, D, k, 0, 5)
    index, q = torch.arange(k, device="cuda").repeat(T, 1) * 100, torch.full((T, k), -1.5, device="cuda")
    index[1], q[2], index[3, 2], index[4, 0] = -1, -float("inf"), V, -2
    dloss = torch.full((T,), 0.25, device="cuda")
    dloss[5] = 0.0
    for normalize in (True, False):
        loss, lse = forward(gs, X, W, index, q, normalize=normalize)
        assert float(loss[1]) == 0 and float(loss[2]) == 0 and bool(torch.isnan(loss[3:5]).all()) and bool(torch.isfinite(loss[5:]).all())
        lse[1], lse[3] = float("nan"), float("inf")
        dX, dW = backward(gs, X, W, index, q, lse, dloss, normalize=normalize)
        silent = [1, 2, 3, 4, 5]
        assert bool((dX[silent] == 0).all()) and bool((dX[[0, 6, 11]] != 0).any(1).all())
        rest = [0] + list(range(6, T))
        alone = backward(gs, X[rest].contiguous(), W, index[rest].contiguous(), q[rest].contiguous(), lse[rest].contiguous(), dloss[rest].contiguous(), normalize=normalize)
        assert torch.equal(alone[0], dX[rest])
    # logits that are not finite, at a token that does not count
    X[1] = float("inf")
    dX, dW = backward(gs, X, W, index, q, lse, dloss, want=(True, False))
    assert bool((dX[1] == 0).all()) and bool(torch.isfinite(dX).all())


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_pieces_of_any_room(gs, dtype):
    T, V, D, k = 130, 5001, 128, 9
    X, W, index, q = inputs(dtype, T, V, D, k, 0, 8)
    loss, lse = forward(gs, X, W, index, q)
    dloss = torch.full((T,), (512.0 if dtype == "f16" else 1.0) / T, device="cuda")
    full = gs.distill_workspace_bytes(dtype, T, V, D, k, backward=True)
    for part in (1.0, 0.6, 0.3):
        dX, dW = backward(gs, X, W, index, q, lse, dloss, room=int(full * part) // 256 * 256)
        check_gradient(dtype, X, W, index, q, 1.0, True, lse, dloss, dX, dW)
    only_x, only_w = backward(gs, X, W, index, q, lse, dloss, want=(True, False))[0], backward(gs, X, W, index, q, lse, dloss, want=(False, True))[1]
    full_x, full_w = backward(gs, X, W, index, q, lse, dloss)
    assert torch.equal(only_x, full_x) and torch.equal(only_w, full_w)
    with pytest.raises(gs.GensorError) as e:
        backward(gs, X, W, index, q, lse, dloss, room=512)
    assert e.value.status == 4


def test_captured_and_replayed(gs):
    T, V, D, k = 77, 2000, 64, 5
    X, W, index, q = inputs("bf16", T, V, D, k, 0, 6)
    loss, lse, dloss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.full((T,), 1.0 / T, device="cuda")
    dX, dW = torch.empty_like(X), torch.empty_like(W)
    ws = workspace(max(gs.distill_workspace_bytes("bf16", T, V, D, k, b) for b in (False, True)))

    def step():
        gs.distill_forward(X, W, index, q, loss, lse, workspace=ws)
        gs.distill_backward(X, W, index, q, lse, dloss, dX, dW, workspace=ws)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (loss, lse, dX, dW)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(3):
        for t in (loss, lse, dX, dW):
            t.fill_(float("nan"))
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((loss, lse, dX, dW), want)), n
        X.neg_()
        graph.replay()
        X.neg_()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_operands_and_gradients_that_start_anywhere(gs, dtype):
    """Rows of any pitch from any element on; what lies around the gradients stays as it is."""
    T, V, D, k = 45, 700, 72, 5
    X, W, index, q = inputs(dtype, T, V, D, k, 0, 31)
    loss, lse = forward(gs, X, W, index, q)
    dloss = torch.full((T,), 1.0 / T, device="cuda")

    def placed(rows, first, pad, values=None):
        flat = torch.full((rows * (D + pad) + 16,), 7.0, device="cuda").to(TORCH[dtype])
        v = flat.as_strided((rows, D), (D + pad, 1), first)
        if values is not None:
            v.copy_(values)
        return flat, v
    for first, pad in ((1, 1), (3, 0), (8, 8)):
        x, w = placed(T, first, pad, X)[1], placed(V, first, pad, W)[1]
        (flat_x, dX), (flat_w, dW) = placed(T, first, pad), placed(V, first, pad)
        out, out_lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        gs.distill_forward(x, w, index, q, out, out_lse, workspace=workspace(gs.distill_workspace_bytes(dtype, T, V, D, k)))
        check_forward(out, out_lse, reference(X, W, index, q, 1.0, True))
        gs.distill_backward(x, w, index, q, out_lse, dloss, dX, dW, workspace=workspace(gs.distill_workspace_bytes(dtype, T, V, D, k, backward=True)))
        check_gradient(dtype, X, W, index, q, 1.0, True, out_lse, dloss, dX, dW)
        for flat, v in ((flat_x, dX), (flat_w, dW)):
            rest = torch.ones_like(flat, dtype=torch.bool)
            rest.as_strided(v.shape, v.stride(), first).fill_(False)
            assert bool((flat[rest] == 7).all())


def test_more_tokens_than_a_launch_has_workgroups_for(gs):
    T, V, D, k = 1_100_003, 7, 3, 2
    X, W, index, q = inputs("f32", T, V, D, k, 0, 41)
    loss, lse = forward(gs, X, W, index, q)
    check_forward(loss, lse, reference(X, W, index, q, 1.0, True))
    dloss = torch.full((T,), 1.0, device="cuda")
    dX, dW = backward(gs, X, W, index, q, lse, dloss)
    check_gradient("f32", X, W, index, q, 1.0, True, lse, dloss, dX, dW)
