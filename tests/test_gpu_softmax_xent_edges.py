"""GPU tests of the softmax cross entropy where its softmax degenerates: nothing beside the target, logits without bounds, logits that are
large and close to each other.  Bounds as derived in test_gpu_softmax_xent.py."""
import math

import numpy as np
import pytest
import torch

from test_gpu_softmax_xent import H, U, backward, buffers, close, forward, mp8, truth  # noqa: F401

pytestmark = pytest.mark.gpu


def tokens(x, w, t):
    """The inputs of a call, halves as given."""
    (M, K), N = x.shape, w.shape[0]
    return dict(M=M, N=N, K=K, ldx=K, ldw=K, x=x.astype(np.float16), w=w.astype(np.float16), t=np.asarray(t, np.int64), dloss=None, x8=False)


def logits(z, N, K=8):
    """Tokens whose first logit is z and whose others are what w's rows make of them: x is one in its first feature."""
    x, w = np.zeros((len(z), K)), np.zeros((N, K))
    x[:, 0], w[0, 0] = 1.0, z[0]
    return x, w


@pytest.mark.parametrize("M", [1, 70, 600])
@pytest.mark.parametrize("z", [-60000.0, -1000.0, -600.0, 0.0, 1000.0])
def test_one_class(mp8, M, z):
    """Nothing stands beside the target: the loss is 0 and lse the logit, wherever it lies, and there is no gradient."""
    x, w = logits([z] * M, 1)
    t = np.zeros(M)
    t[1::5] = -1
    c = tokens(x, w, t)
    x, w, t, loss, lse = forward(mp8, c)
    live = t == 0
    assert not loss.any()
    assert bool((lse[live] == z).all()) and bool(((lse - z).abs() <= 4 * U * abs(z)).all())
    dx, dw = buffers(M, 1, 8, torch.float16)
    stats = mp8.new_stats()
    backward(mp8, c, x, w, t, loss, lse, scale=1024.0, dx16=dx[:M * 8], dw16=dw[:8], dx_stats=stats, dw_stats=stats)
    assert not dx[:M * 8].any() and not dw[:8].any() and mp8.read_stats(stats) == (0, 0, 0)


def test_other_classes_without_probability(mp8):
    """Logits of minus infinity beside the target's."""
    for z in (-1000.0, -2.0, 1000.0):
        x, w = logits([z] * 3, 200)
        w[1:, 0] = -np.inf
        loss, lse = forward(mp8, tokens(x, w, [0, 0, 0]))[3:]
        assert not loss.any() and bool((lse == z).all())


def test_infinite_logits(mp8):
    """From the definition: a target at minus infinity leaves lse to the others (its loss is infinite), one at plus infinity has no loss, and a
    row of nothing but infinities has none either; what is not a number stays so, whichever class it is."""
    N, inf = 300, np.inf
    rng = np.random.default_rng(2)
    w = np.zeros((N, 8))
    w[:, 0] = rng.standard_normal(N)
    w = w.astype(np.float16).astype(np.float64)
    w[0, 0], w[1, 0], w[2, 0] = inf, -inf, np.nan
    x = np.zeros((1, 8))
    x[0, 0] = 1.0
    usual = [k for k in range(3, N)]
    # classes, target among them, loss, lse
    others = lambda keep: float(np.log(np.exp(w[keep, 0]).sum()))
    for keep, target, loss, lse in ((usual, 5, others(usual) - w[usual[5], 0], others(usual)), (usual + [1], 5, others(usual) - w[usual[5], 0], others(usual)),
                                    (usual + [1], len(usual), inf, others(usual)), (usual + [0], len(usual), np.nan, inf), ([0], 0, np.nan, inf),
                                    ([1], 0, np.nan, -inf), (usual + [2], 5, np.nan, np.nan), (usual + [2], len(usual), np.nan, np.nan), ([2], 0, np.nan, np.nan)):
        got = forward(mp8, tokens(x, w[keep], [target]))
        r = (math.log(2) * 12 + 64 + N / 32 + 16) * U  # (products with zeros and one are exact)
        for value, want, bound in ((float(got[3]), loss, r * abs(loss)), (float(got[4]), lse, r + 4 * U * abs(lse))):
            if np.isfinite(want):
                assert abs(value - want) <= bound, (target, value, want)
            else:
                assert value == want or (np.isnan(value) and np.isnan(want)), (target, value, want)


@pytest.mark.parametrize("common", [0.0, 2.0 ** 10, -2.0 ** 14, 2.0 ** 17, -2.0 ** 17])
@pytest.mark.parametrize("M,N", [(3, 40), (130, 700), (700, 3000)])
def test_a_part_that_all_logits_have_in_common_cancels(mp8, common, M, N):
    """Logits in steps of 2^-6, exact in FP32 whatever they have in common (dz = 0), so that only the softmax's own roundings are left.  Differences
    are scaled by an FP32 log2 e on one side and undone on the other: that is one more U of the spread."""
    rng = np.random.default_rng(N)
    x, w = np.zeros((M, 8)), np.zeros((N, 8))
    x[:, 0], w[:, 0] = 512.0, common / 512.0
    x[:, 1:3] = rng.integers(-2, 3, (M, 2))
    w[:, 1:3] = rng.integers(-64, 65, (N, 2)) / 64.0
    c = tokens(x, w, rng.integers(0, N, M))
    z = x @ w.T
    assert (z == z.astype(np.float32)).all()
    want = truth(c)
    r = (2 * math.log(2) * ((z.max(1) - z.min(1)) / math.log(2) + 1) + 64 + N / 32 + 16) * U
    loss, lse = forward(mp8, c)[3:]
    close(loss, want["loss"], want["loss"] * (r + 4 * U), "loss")
    close(lse, want["lse"], r + 4 * U * np.abs(want["lse"]), "lse")


@pytest.mark.parametrize("M,N,K", [(1 << 20, 1 << 19, 64), ((1 << 18) - 77, 1 << 21, 8)])
def test_as_many_logits_as_a_launch_takes(mp8, M, N, K):
    """About 2^23 tiles of 256x256, 2^39 logits: some tokens from all over, the last ones among them."""
    import test_gpu_operator_tiles as tiles
    x, w, t = tiles.inputs(1, M, N, K)
    t[-1], t[-2] = N - 1, -1
    loss, lse = torch.full((M,), 7.0, device="cuda"), torch.full((M,), 7.0, device="cuda")
    mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=torch.empty(mp8.softmax_xent_fwd_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda"))
    rows = torch.cat([torch.arange(0, M, M // 16, device="cuda"), torch.arange(M - 8, M, device="cuda")])
    want = tiles.truth(x[rows].double(), w.double(), t[rows], 1.0)
    tiles.within(lse[rows], want["lse"], want["dlse"], "lse")
    tiles.within(loss[rows], want["loss"], want["loss"] * (want["r"] + 4 * U) + 1e-44, "loss")
    assert bool((loss >= 0).all()) and bool(((lse > 0) & (lse < 100)).all())  # (every token has been written)


@pytest.mark.parametrize("common", [0.0, 2.0 ** 10, -2.0 ** 14, 2.0 ** 17])
def test_gradient_of_logits_with_a_common_part(mp8, common):
    """The gradient's probabilities are exp(z - lse) with lse, its product with log2 e and their difference from the token weight's exponent in
    FP32: 3 U |lse|, and 64 U for a shift of up to 64, beside what the loss has (the target's comes from the loss itself)."""
    M, N = 130, 700
    rng = np.random.default_rng(N)
    x, w = np.zeros((M, 8)), np.zeros((N, 8))
    x[:, 0], w[:, 0] = 512.0, common / 512.0
    x[:, 1:3] = rng.integers(-2, 3, (M, 2))
    w[:, 1:3] = rng.integers(-64, 65, (N, 2)) / 64.0
    t = rng.integers(0, N, M)
    c = tokens(x, w, t)
    z = x @ w.T
    lse = z.max(1) + np.log(np.exp(z - z.max(1)[:, None]).sum(1))
    loss = truth(c)["loss"]
    e = np.exp(z - lse[:, None])
    e[np.arange(M), t] = np.expm1(-loss)
    r = (2 * math.log(2) * ((z.max(1) - z.min(1)) / math.log(2) + 1) + 64 + N / 32 + 16) * U
    de = (H + r + 64 * U + 3 * U * np.abs(lse))[:, None] * np.abs(e) + 2.0 ** -39
    x, w = np.abs(x), np.abs(w)
    dev = forward(mp8, c)
    dx, dw = buffers(M, N, 8, torch.float16)
    backward(mp8, c, *dev, dx16=dx[:M * 8], dw16=dw[:N * 8])
    for got, want, bound, what in ((dx[:M * 8], e @ c["w"].astype(np.float64), de @ w + N * U * (np.abs(e) @ w), "dx"),
                                   (dw[:N * 8], e.T @ c["x"].astype(np.float64), de.T @ x + M * U * (np.abs(e).T @ x), "dw")):
        close(got, want, bound + H * (np.abs(want) + bound) + 2.0 ** -25, what)
