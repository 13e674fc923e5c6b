"""GPU tests of mp8_orthogonal_momentum_fp16_sr against its definition in 64 bits.

The velocity is exact.  The direction X is the Newton-Schulz iteration on half operands: what it may be off by comes from a model of
the roundings (`rounded` below: the iterates, A and the polynomial each rounded once to half at their scales, everything else in 64
bits), not from the kernel.  Kernel and model round the same quantities, whose FP32 sums differ in their last bits only, so that the kernel
is about as far from the exact iteration as the model is: asserted to within twice that and a rounding to half of the result."""
import math

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315
U, H = 2.0 ** -24, 2.0 ** -11


@pytest.fixture(scope="module")
def mp8():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1905_12334_amd as m
    m.lib()
    return m


def iterate(u, steps, rounded):
    """X after `steps`; `rounded`: with the operands rounded to half as stored (X times s, A and the polynomial times 2^14)."""
    tall = u.shape[0] > u.shape[1]
    u = u.T if tall else u
    norm = np.linalg.norm(u)
    x = u / norm if norm else u * 0
    s = 2.0 ** np.rint(0.5 * math.log2(u.shape[1]))
    half = (lambda v, f: (v * f).astype(np.float16).astype(np.float64) / f) if rounded else (lambda v, f: v)
    x = half(x, s)
    for k in range(steps):
        a = half(x @ x.T, 2.0 ** 14)
        p = half(B * a + C * (a @ a), 2.0 ** 14)
        x = A * x + p @ x
        if k + 1 < steps:
            x = half(x, s)
    return x.T if tall else x


def gradient(rng, rows, cols, kind="noise"):
    g = rng.standard_normal((rows, cols))
    if kind == "strong":
        r = max(1, min(rows, cols) // 16)
        g = 0.2 * g + rng.standard_normal((rows, r)) @ rng.standard_normal((r, cols)) / math.sqrt(r)
    return g


def run(mp8, w, v, g8, lr, inv, mu, **kw):
    dev = [torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in (w, v, g8)]
    shape = w.shape
    batch = int(np.prod(shape[:-2], dtype=np.int64))
    ws = torch.full((max(16, mp8.orthogonal_momentum_workspace_bytes(batch, *shape[-2:])),), 0xFF, dtype=torch.uint8, device="cuda")
    mp8.orthogonal_momentum_fp16_sr(dev[0], dev[1], dev[2], lr, inv, mu, workspace=ws, **kw)
    return dev[0].cpu().numpy(), dev[1].cpu().numpy()


def direction(v, g, mu, nesterov):
    v, g = v.astype(np.float64), g.astype(np.float64)
    return g + mu * v if nesterov else v


def velocity(v, g8, inv, mu):
    """As mp8_sgd_momentum_fp16_sr: the oracle's, with weights of zero."""
    n = v.size
    return oracle.sgd_momentum_fp16(np.zeros(n, np.uint16), v.reshape(-1).copy(), g8.reshape(-1), 0.0, inv, mu, 0.0)[1].reshape(v.shape)


def codes(x):
    return oracle.quantize_e5m2(np.ascontiguousarray(x, np.float32).reshape(x.shape[0], -1))[0].reshape(x.shape)


def values(c):
    return (c.astype(np.uint16) << 8).view(np.float16).astype(np.float64)


SHAPES = [(1, 1), (1, 9), (7, 1), (8, 8), (5, 64), (64, 64), (65, 63), (72, 200), (200, 72), (128, 1152), (1152, 128), (130, 131),
          (250, 1000), (333, 257), (512, 512), (1000, 520), (700, 1500)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("kind", ["noise", "strong"])
def test_direction_against_64_bits(mp8, rows, cols, kind):
    rng = np.random.default_rng(rows * 31 + cols)
    g8 = codes(gradient(rng, rows, cols, kind))
    v = (gradient(rng, rows, cols, kind) * 0.5).astype(np.float32)
    mu, inv, nesterov = 0.95, 0.5, cols % 2 == 0
    w16, got_v = run(mp8, np.zeros((rows, cols), np.float16), v, g8, -1.0, inv, mu, nesterov=nesterov, round=mp8.RNE)
    want_v = velocity(v, g8, inv, mu)
    assert np.array_equal(got_v.view(np.uint32), want_v.view(np.uint32))
    u = direction(want_v, values(g8) * inv, np.float32(mu).astype(np.float64), nesterov)
    exact, model = iterate(u, 5, False), iterate(u, 5, True)
    norm = np.linalg.norm(exact)
    tolerance = 2 * np.linalg.norm(model - exact) + H * norm
    off = np.linalg.norm(w16.astype(np.float64) - exact)
    assert off <= tolerance, (off / norm, tolerance / norm)
    if min(rows, cols) > 1 and kind == "noise":
        s = np.linalg.svd(w16.astype(np.float64), compute_uv=False)
        assert s.max() < 1.25


@pytest.mark.parametrize("steps", [1, 2, 7])
def test_number_of_steps(mp8, steps):
    rng = np.random.default_rng(steps)
    g8 = codes(gradient(rng, 90, 140))
    w16, v = run(mp8, np.zeros((90, 140), np.float16), np.zeros((90, 140), np.float32), g8, -1.0, 1.0, 0.9, steps=steps, nesterov=False, round=mp8.RNE)
    u = values(g8)
    exact, model = iterate(u, steps, False), iterate(u, steps, True)
    assert np.linalg.norm(w16 - exact) <= 2 * np.linalg.norm(model - exact) + H * np.linalg.norm(exact)


@pytest.mark.parametrize("rows,cols", [(96, 160), (161, 93)])
@pytest.mark.parametrize("sr", [False, True])
def test_update_of_the_weights(mp8, rows, cols, sr):
    """w' is half(fma(-lr, fma(wd, w, X), w)): with X as the kernel has it (taken from a call on zero weights, exact to a half's
    rounding), rounding of an interval of lr * (2^-11 |X| + 2^-25) and FP32's own; stochastic rounding is monotone for an element's own bits."""
    rng = np.random.default_rng(3)
    g8, v = codes(gradient(rng, rows, cols)), np.zeros((rows, cols), np.float32)
    x = run(mp8, np.zeros((rows, cols), np.float16), v, g8, -1.0, 1.0, 0.9, round=mp8.RNE)[0].astype(np.float64)
    w = (rng.standard_normal((rows, cols)) * 0.05).astype(np.float16)
    lr, wd = np.float32(0.03), np.float32(0.1)
    w8 = torch.full((rows * cols + 64,), 0xAA, dtype=torch.uint8, device="cuda")
    got, _ = run(mp8, w, v, g8, float(lr), 1.0, 0.9, weight_decay=float(wd), round=mp8.SR if sr else mp8.RNE, seed=77, offset=9,
                 w8_out=w8[:rows * cols])
    wide = w.astype(np.float64)
    new = wide - float(lr) * (x + float(wd) * wide)
    slack = float(lr) * (H * np.abs(x) + 2.0 ** -25) + 4 * U * np.abs(wide)
    assert bool((w8[rows * cols:] == 0xAA).all())

    def rounded(val):
        h = oracle.fp16_encode_array(val.astype(np.float32).reshape(-1), mode=oracle.SR if sr else oracle.RNE, seed=77, offset=9)
        return np.asarray(h, np.uint16).view(np.float16).reshape(val.shape)
    lo, hi = rounded(new - slack), rounded(new + slack)
    assert ((lo <= got) & (got <= hi)).all()
    want8 = oracle.quantize_e5m2(got.astype(np.float32))[0]
    assert np.array_equal(w8[:rows * cols].cpu().numpy(), want8.reshape(-1))


def test_every_matrix_of_a_batch_by_itself(mp8):
    """Also where one of them is zero (its direction is zero) and one has an Inf (it alone becomes NaN)."""
    rng = np.random.default_rng(8)
    for rows, cols in ((40, 72), (75, 33), (33, 35)):
        n, mu, inv = 6, 0.9, 0.5
        g8 = np.stack([codes(gradient(rng, rows, cols)) for _ in range(n)])
        v = (rng.standard_normal((n, rows, cols)) * 0.3).astype(np.float32)
        g8[2], v[2] = 0, 0
        g8[4, 3, 5] = 0x7C
        stats = mp8.new_stats()
        got_w, got_v = run(mp8, np.zeros((n, rows, cols), np.float16), v, g8, -1.0, inv, mu, round=mp8.RNE, stats=stats)
        assert mp8.read_stats(stats)[1] == 1
        assert np.isnan(got_w[4]).all() and not got_w[2].any()
        for i in (0, 1, 3, 5):
            want_v = velocity(v[i], g8[i], inv, mu)
            assert np.array_equal(got_v[i].view(np.uint32), want_v.view(np.uint32))
            u = direction(want_v, values(g8[i]) * inv, np.float32(mu).astype(np.float64), True)
            exact, model = iterate(u, 5, False), iterate(u, 5, True)
            assert np.linalg.norm(got_w[i] - exact) <= 2 * np.linalg.norm(model - exact) + H * np.linalg.norm(exact)


@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e-4, 1e10, 1e25])
def test_gradients_of_any_size(mp8, size):
    rng = np.random.default_rng(2)
    rows, cols = 48, 80
    g8 = np.zeros((rows, cols), np.uint8)
    v = gradient(rng, rows, cols)
    zero = np.zeros((rows, cols), np.float16)
    a = run(mp8, zero, (v * size).astype(np.float32), g8, -1.0, 1.0, 1.0, nesterov=False, round=mp8.RNE)[0]
    u = (v * size).astype(np.float32).astype(np.float64)
    exact, model = iterate(u, 5, False), iterate(u, 5, True)
    assert np.linalg.norm(a - exact) <= 2 * np.linalg.norm(model - exact) + H * np.linalg.norm(exact)


def test_a_skipped_step_changes_nothing_and_counts(mp8):
    rng = np.random.default_rng(4)
    rows, cols = 70, 90
    g8 = codes(gradient(rng, rows, cols))
    g8[1, 2] = 0x7F
    v, w = rng.standard_normal((rows, cols)).astype(np.float32), (rng.standard_normal((rows, cols)) * 0.1).astype(np.float16)
    for flag, count in ((1, True), (7, False), (0, True)):
        skip = torch.tensor([flag], dtype=torch.int32, device="cuda")
        w8 = torch.full((rows * cols,), 0xAA, dtype=torch.uint8, device="cuda")
        stats = mp8.new_stats() if count else None
        got_w, got_v = run(mp8, w, v, g8, 0.1, 1.0, 0.9, skip_if_nonzero=skip, w8_out=w8, stats=stats)
        if count:
            assert mp8.read_stats(stats)[1] == 1
        if flag:
            assert np.array_equal(got_w, w) and np.array_equal(got_v, v) and bool((w8 == 0xAA).all())
        else:
            assert np.isnan(got_w).all()


def test_results_repeat_and_a_captured_step_replays(mp8):
    rng = np.random.default_rng(5)
    shape = (3, 100, 260)
    g8 = torch.from_numpy(codes(gradient(rng, 300, 260)).reshape(shape)).cuda()
    w0 = torch.from_numpy((rng.standard_normal(shape) * 0.1).astype(np.float16)).cuda()
    v0 = torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()
    ws = torch.empty(mp8.orthogonal_momentum_workspace_bytes(*shape), dtype=torch.uint8, device="cuda")

    def steps(w, v, n):
        for k in range(n):
            mp8.orthogonal_momentum_fp16_sr(w, v, g8, 0.02, 0.5, 0.95, seed=1, offset=2, workspace=ws)
    w, v = w0.clone(), v0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps(w, v, 1)
    ew, ev = w0.clone(), v0.clone()
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        seen = w.clone(), v.clone()
        ws.fill_(0xFF)
        steps(ew, ev, 1)
        torch.cuda.synchronize()
        assert torch.equal(seen[0], ew) and torch.equal(seen[1], ev)


def test_zero_dimensions_do_nothing(mp8):
    e = lambda d: torch.empty((2, 0, 5), dtype=d, device="cuda")
    mp8.orthogonal_momentum_fp16_sr(e(torch.float16), e(torch.float32), e(torch.uint8), 0.1, 1.0, 0.9)
    assert mp8.orthogonal_momentum_workspace_bytes(0, 4, 4) == mp8.orthogonal_momentum_workspace_bytes(1, 0, 4) == 0
