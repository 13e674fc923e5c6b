"""GPU tests of the softmax cross entropy (mp8_softmax_xent_fwd_fp16 / _bwd_fp16) against its definition in 64 bits.

Tolerances, from the arithmetic.  u = 2^-24 is half a step of FP32, h = 2^-11 of a half.
  logits    a chain of at most K additions in FP32:  |dz| <= K u sum|x||w|
  softmax   an exponent's argument, at most `spread` powers of two below the largest, is rounded once and the sums are chains of at
            most 64 + N / 32 additions: relative error r = 2 max|dz| + (ln 2 * spread + 64 + N / 32 + 16) u, of the sum, of a
            probability, and (because q / (1 + q) <= log(1 + q)) of the loss
  error e   rounded to half, times 2^14 over the largest weight's power of two: h |e| and 2^-39 of the largest weight
  gradient  what the errors of e become in a sum of |e||w|, FP32 additions, and one rounding (h, subnormals 2^-25)
The elementwise bound adds every term's largest error.  As a whole (2-norm) the two roundings to half are independent and
uniform: h / sqrt 3 each, together 0.82 h, asserted as h."""
import math

import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -11


@pytest.fixture(scope="module")
def mp8():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1905_12334_amd as m
    m.lib()
    return m


def case(seed, M, N, K, x8=False, ldx=None, ldw=None, ignored=0.0, peak=4.0, weighted=False):
    """Inputs on the host.  What lies behind a row's K elements is NaN."""
    rng = np.random.default_rng(seed)
    ldx, ldw = ldx or K, ldw or K
    w = (rng.standard_normal((N, K)) * K ** -0.5).astype(np.float16)
    t = rng.integers(0, N, M)
    x = (rng.standard_normal((M, K)) + peak * rng.random((M, 1)) * w[t].astype(np.float32)).astype(np.float16)
    if x8:
        x = oracle.quantize_e5m2(x.astype(np.float32))[0]
    for k, i in enumerate(np.nonzero(rng.random(M) < ignored)[0]):
        t[i] = (-100, -1, N, N + 5)[k % 4]
    xs = np.full((M, ldx), 0x7F if x8 else np.nan, np.uint8 if x8 else np.float16)
    ws = np.full((N, ldw), np.nan, np.float16)
    xs[:, :K], ws[:, :K] = x, w
    d = (rng.random(M) * 2 - 0.5).astype(np.float32) if weighted else None
    return dict(M=M, N=N, K=K, ldx=ldx, ldw=ldw, x=xs, w=ws, t=t.astype(np.int64), dloss=d, x8=x8)


def half_of_codes(c):
    return (c.astype(np.uint16) << 8).view(np.float16)


def truth(c, scale=1.0):
    """Results and elementwise bounds in 64 bits."""
    M, N, K = c["M"], c["N"], c["K"]
    x = c["x"][:, :K]
    x = (half_of_codes(x) if c["x8"] else x).astype(np.float64)
    w, t = c["w"][:, :K].astype(np.float64), c["t"]
    live = (t >= 0) & (t < N)
    at = np.where(live, t, 0)
    rows = np.arange(M)
    with np.errstate(all="ignore"):
        z = x @ w.T
        dz = K * U * (np.abs(x) @ np.abs(w).T).max(1)
        top = z.max(1)
        total = np.exp(z - top[:, None]).sum(1)
        lse = top + np.log(total)
        behind = z - z[rows, at][:, None]
        others = np.exp(behind)
        others[rows, at] = 0
        loss = np.where(live, np.log1p(others.sum(1)), 0.0)
        spread = (top - z.min(1)) / math.log(2) + 1
        r = 2 * dz + (math.log(2) * spread + 64 + N / 32 + 16) * U
        p = np.exp(z - lse[:, None])
        p[rows, at] -= live
        p[rows[live], t[live]] = np.expm1(-loss[live])
    f = np.where(live, scale * (c["dloss"].astype(np.float64) if c["dloss"] is not None else 1.0), 0.0)
    x = np.where(live[:, None], x, 0.0)
    e = np.where(live[:, None], p, 0.0) * f[:, None]
    dlse = r + 4 * U * np.abs(lse)  # (of tokens without a target too)
    r = np.where(live, r, 0.0)
    largest = np.abs(f).max() if M else 0.0
    de = (H + r + 8 * U)[:, None] * np.abs(e) + 2.0 ** -39 * largest
    de = np.where(live[:, None], de, 0.0)
    dx, dw = e @ w, e.T @ x
    bx = de @ np.abs(w) + N * U * (np.abs(e) @ np.abs(w))
    bw = de.T @ np.abs(x) + M * U * (np.abs(e).T @ np.abs(x))
    return dict(loss=loss, lse=lse, dx=dx, dw=dw, bx=bx + H * (np.abs(dx) + bx) + 2.0 ** -25, bw=bw + H * (np.abs(dw) + bw) + 2.0 ** -25,
                r=r, dlse=dlse, live=live)


def forward(mp8, c, ws=None):
    x, w, t = (torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (c["x"], c["w"], c["t"]))
    M, N, K = c["M"], c["N"], c["K"]
    loss, lse = torch.full((M + 8,), 7.0, device="cuda"), torch.full((M + 8,), 7.0, device="cuda")
    if ws is None:
        ws = torch.full((max(16, mp8.softmax_xent_fwd_workspace_bytes(M, N, K, c["ldw"])),), 0xFF, dtype=torch.uint8, device="cuda")
    mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss[:M], lse[:M], workspace=ws, ldx=c["ldx"], ldw=c["ldw"])
    assert bool((loss[M:] == 7).all()) and bool((lse[M:] == 7).all()), "wrote behind the last token"
    return x, w, t, loss[:M], lse[:M]


def backward(mp8, c, x, w, t, loss, lse, ws=None, **kw):
    M, N, K = c["M"], c["N"], c["K"]
    if ws is None:
        ws = torch.full((mp8.softmax_xent_bwd_workspace_bytes(M, N, K, c["ldw"]),), 0xFF, dtype=torch.uint8, device="cuda")
    d = torch.from_numpy(c["dloss"]).cuda() if c["dloss"] is not None else None
    mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dloss=d, workspace=ws, ldx=c["ldx"], ldw=c["ldw"], **kw)


def buffers(M, N, K, dtype):
    fill = 0xAA if dtype == torch.uint8 else 7.0
    return [torch.full((n * K + 64,), fill, dtype=dtype, device="cuda") for n in (M, N)]


def close(got, want, bound, what):
    got = got.double().cpu().numpy().reshape(want.shape)
    off = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (off <= bound).all(), (what, float((off / bound).max()))


def norm_off(got, want):
    got = got.double().cpu().numpy().reshape(want.shape)
    n = np.linalg.norm(want)
    return np.linalg.norm(got - want) / n if n else np.abs(got).max(initial=0.0)


SHAPES = [
    (1, 1, 1), (1, 2, 8), (1, 1000, 512), (3, 7, 5), (2, 64, 64), (17, 65, 72), (64, 64, 128), (65, 129, 136), (128, 128, 192),
    (200, 333, 100), (256, 1000, 2048), (33, 5003, 200), (700, 1030, 264), (1030, 2100, 520), (2100, 70, 80), (5000, 3, 33)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_loss_and_gradient_against_64_bits(mp8, M, N, K):
    c = case(M * 7 + N, M, N, K, ignored=0.2 if M > 2 else 0.0, weighted=M % 2 == 1)
    scale = 64.0 / M
    want = truth(c, scale)
    x, w, t, loss, lse = forward(mp8, c)
    close(lse, want["lse"], want["dlse"], "lse")
    close(loss, want["loss"], want["loss"] * (want["r"] + 4 * U) + 1e-44, "loss")
    dx, dw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, scale=scale, dx16=dx[:M * K], dw16=dw[:N * K])
    assert bool((dx[M * K:] == 7).all()) and bool((dw[N * K:] == 7).all())
    close(dx[:M * K], want["dx"], want["bx"], "dx")
    close(dw[:N * K], want["dw"], want["bw"], "dw")
    if M * K > 4000 and N > 50:
        assert norm_off(dx[:M * K], want["dx"]) <= H and norm_off(dw[:N * K], want["dw"]) <= H
    assert not dx[:M * K].view(M, K)[torch.from_numpy(~want["live"]).cuda()].any()


@pytest.mark.parametrize("M,N,K,ldx,ldw", [(70, 130, 64, 72, 80), (70, 130, 64, 67, 71), (40, 90, 61, 61, 64), (300, 600, 96, 96, 97), (9, 20, 7, 16, 8)])
@pytest.mark.parametrize("x8", [False, True])
def test_leading_dimensions_and_what_lies_behind_the_rows(mp8, M, N, K, ldx, ldw, x8):
    c = case(5, M, N, K, x8=x8, ldx=ldx, ldw=ldw, ignored=0.1)
    want = truth(c, 2.0)
    x, w, t, loss, lse = forward(mp8, c)
    close(lse, want["lse"], want["dlse"], "lse")
    dx, dw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, scale=2.0, dx16=dx[:M * K], dw16=dw[:N * K])
    close(dx[:M * K], want["dx"], want["bx"], "dx")
    close(dw[:N * K], want["dw"], want["bw"], "dw")


def test_gradient_against_differences(mp8):
    """d loss / d x and d w by central differences of the definition in 64 bits (step 1e-4: error 1e-8 of the third derivative)."""
    M, N, K = 5, 11, 9
    c = case(3, M, N, K, weighted=True)
    c["t"][1] = -1
    x, w, t, loss, lse = forward(mp8, c)
    dx, dw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, scale=8.0, dx16=dx[:M * K], dw16=dw[:N * K])
    live = c["t"] >= 0

    def total(xs, ws):
        z = xs @ ws.T
        l = np.log(np.exp(z).sum(1)) - z[np.arange(M), np.where(live, c["t"], 0)]
        return 8.0 * (c["dloss"].astype(np.float64) * l)[live].sum()
    xs, ws = c["x"].astype(np.float64), c["w"].astype(np.float64)
    want = truth(c, 8.0)
    for got, arr, bound in ((dx[:M * K], xs, want["bx"]), (dw[:N * K], ws, want["bw"])):
        got = got.double().cpu().numpy().reshape(arr.shape)
        for i in np.ndindex(arr.shape):
            keep = arr[i]
            arr[i] = keep + 1e-4
            up = total(xs, ws)
            arr[i] = keep - 1e-4
            down = total(xs, ws)
            arr[i] = keep
            assert abs(got[i] - (up - down) / 2e-4) <= bound[i] + 1e-6, i


def test_the_loss_keeps_its_precision_near_zero(mp8):
    M, N, K = 64, 500, 64
    c = case(9, M, N, K)
    w = c["w"].astype(np.float64)
    c["x"] = (np.random.default_rng(1).uniform(5, 40, (M, 1)) * w[c["t"]]).astype(np.float16)
    want = truth(c, 1.0)
    assert want["loss"].min() < 1e-9
    x, w, t, loss, lse = forward(mp8, c)
    close(loss, want["loss"], want["loss"] * (want["r"] + 4 * U), "loss")
    dx, dw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, scale=1.0, dx16=dx[:M * K], dw16=dw[:N * K])
    close(dx[:M * K], want["dx"], want["bx"], "dx")


def test_tokens_without_a_target_may_hold_anything(mp8):
    M, N, K = 150, 300, 128
    c = case(4, M, N, K, ignored=0.3, weighted=True)
    live = (c["t"] >= 0) & (c["t"] < N)
    dirty = dict(c, x=c["x"].copy(), dloss=c["dloss"].copy())
    bad = np.nonzero(~live)[0]
    for k, i in enumerate(bad):
        dirty["x"][i] = (np.nan, np.inf, -np.inf, 65504.0)[k % 4]
        dirty["dloss"][i] = (np.inf, np.nan)[k % 2]
    outs = []
    for d in (c, dirty):
        x, w, t, loss, lse = forward(mp8, d)
        dx, dw = buffers(M, N, K, torch.float16)
        backward(mp8, d, x, w, t, loss, lse, scale=4.0, dx16=dx[:M * K], dw16=dw[:N * K])
        outs.append((loss.clone(), dx, dw))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    # no target at all
    c["t"][:] = -100
    x, w, t, loss, lse = forward(mp8, c)
    close(lse, truth(c)["lse"], truth(c)["dlse"], "lse")
    dx, dw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, dx16=dx[:M * K], dw16=dw[:N * K])
    assert not loss.any() and not dx[:M * K].any() and not dw[:N * K].any()


def test_nan_in_a_token_stays_in_its_row_and_in_the_weights_gradient(mp8):
    M, N, K = 80, 90, 64
    c = case(6, M, N, K)
    c["x"][7, 3] = np.nan
    x, w, t, loss, lse = forward(mp8, c)
    assert bool(torch.isnan(lse[7])) and bool(torch.isnan(loss[7])) and int(torch.isnan(loss).sum()) == 1
    dx, dw = buffers(M, N, K, torch.float16)
    stats = mp8.new_stats()
    backward(mp8, c, x, w, t, loss, lse, dx16=dx[:M * K], dw16=dw[:N * K], dw_stats=stats)
    nan = torch.isnan(dx[:M * K].view(M, K))
    assert bool(nan[7].all()) and int(nan.sum()) == K
    assert bool(torch.isnan(dw[:N * K]).all())
    assert mp8.read_stats(stats)[:2] == (0x7FC00000, N * K)


@pytest.mark.parametrize("spread", [2.0 ** -30, 2.0 ** -10, 1.0, 2.0 ** 40])
def test_weights_of_any_size(mp8, spread):
    """A common factor of the weights changes nothing but the scale; weights of zero switch tokens off."""
    M, N, K = 64, 200, 64
    c = case(8, M, N, K, weighted=True)
    c["dloss"] = (c["dloss"] * np.float32(spread)).astype(np.float32)
    c["dloss"][5] = 0.0
    scale = 16.0 / spread
    want = truth(c, scale)
    x, w, t, loss, lse = forward(mp8, c)
    dx, dw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, scale=scale, dx16=dx[:M * K], dw16=dw[:N * K])
    close(dx[:M * K], want["dx"], want["bx"], "dx")
    close(dw[:N * K], want["dw"], want["bw"], "dw")
    assert not dx[5 * K:6 * K].any()


@pytest.mark.parametrize("sr", [False, True])
@pytest.mark.parametrize("M,N,K", [(130, 200, 96), (50, 77, 37)])
def test_eight_bit_gradients(mp8, M, N, K, sr):
    """Codes are the rounding of a value within the FP32 bound of the true one: a neighbour of an interval, and with stochastic rounding
    the one the element's own 16 bits choose."""
    c = case(11, M, N, K, ignored=0.1)
    scale = 2.0 ** 10
    want = truth(c, scale)
    x, w, t, loss, lse = forward(mp8, c)
    kw = dict(scale=scale, round=mp8.SR if sr else mp8.RNE, seed=0x1234567890, dx_offset=5, dw_offset=6)
    dx, dw = buffers(M, N, K, torch.uint8)
    hx, hw = buffers(M, N, K, torch.float16)
    sx, sw = mp8.new_stats(), mp8.new_stats()
    backward(mp8, c, x, w, t, loss, lse, dx8=dx[:M * K], dw8=dw[:N * K], dx16=hx[:M * K], dw16=hw[:N * K], dx_stats=sx, dw_stats=sw, **kw)
    assert bool((dx[M * K:] == 0xAA).all()) and bool((dw[N * K:] == 0xAA).all())
    for codes, value, bound, offset, stats, n in ((dx, want["dx"], want["bx"], 5, sx, M * K), (dw, want["dw"], want["bw"], 6, sw, N * K)):
        got = codes[:n].cpu().numpy()
        mode = oracle.SR if sr else oracle.RNE
        # (rounding is monotone for an element's bits)
        lo = oracle.quantize_e5m2((value - bound).astype(np.float32), mode=mode, seed=0x1234567890, offset=offset)[0].reshape(-1)
        hi = oracle.quantize_e5m2((value + bound).astype(np.float32), mode=mode, seed=0x1234567890, offset=offset)[0].reshape(-1)
        f = lambda a: half_of_codes(a).astype(np.float64)
        assert ((f(lo) <= f(got)) & (f(got) <= f(hi))).all()
        amax, nonfinite, zeroed = mp8.read_stats(stats)
        top = np.abs(value).max()
        assert nonfinite == 0 and abs(np.uint32(amax).view(np.float32) - top) <= bound.max()
        assert zeroed <= int((got & 0x7F == 0).sum())
    # half results do not depend on what else is asked for
    ax, aw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, dx16=ax[:M * K], **kw)
    backward(mp8, c, x, w, t, loss, lse, dw16=aw[:N * K], **kw)
    assert torch.equal(ax, hx) and torch.equal(aw, hw)


def test_overflow_is_counted(mp8):
    M, N, K = 40, 50, 64
    c = case(12, M, N, K)
    x, w, t, loss, lse = forward(mp8, c)
    for dtype, key in ((torch.uint8, "8"), (torch.float16, "16")):
        dx, dw = buffers(M, N, K, dtype)
        stats = mp8.new_stats()
        backward(mp8, c, x, w, t, loss, lse, scale=2.0 ** 24, dx_stats=stats, **{"dx" + key: dx[:M * K], "dw" + key: dw[:N * K]})
        got = dx[:M * K].view(torch.float8_e5m2).float() if dtype == torch.uint8 else dx[:M * K].float()
        assert mp8.read_stats(stats)[1] == int((~torch.isfinite(got)).sum()) > 0
    sat, _ = buffers(M, N, K, torch.uint8)
    stats = mp8.new_stats()
    backward(mp8, c, x, w, t, loss, lse, scale=2.0 ** 24, flags=mp8.FLAG_SATURATE, dx8=sat[:M * K], dx_stats=stats)
    assert mp8.read_stats(stats)[1] == 0 and bool(torch.isfinite(sat[:M * K].view(torch.float8_e5m2).float()).all())


def test_many_pieces_of_the_vocabulary(mp8):
    """More classes than one piece of the backward pass holds (512 MB of e): against autograd in FP32 on the GPU,
    whose own error (1e-6) is far below the bound h."""
    M, N, K = 40000, 9000, 64
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = (torch.randn((N, K), generator=gen, device="cuda") * K ** -0.5).half()
    x = torch.randn((M, K), generator=gen, device="cuda").half()
    t = torch.randint(0, N, (M,), generator=gen, device="cuda")
    t[-1000:] = -1
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    need = mp8.softmax_xent_bwd_workspace_bytes(M, N, K)
    assert need < 2 * M * N, "meant to take several pieces"
    ws = torch.empty(max(need, mp8.softmax_xent_fwd_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=ws)
    mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dx16=dx, dw16=dw, scale=1.0, workspace=ws)
    z = x.float() @ w.float().t()
    ref = torch.logsumexp(z, 1)
    assert float((lse - ref).abs().max()) < 1e-5
    e = torch.exp(z - ref[:, None])
    e[torch.arange(M), t.clamp(min=0)] -= 1
    e[-1000:] = 0
    for got, want in ((dx, e @ w.float()), (dw, e.t().contiguous() @ x.float())):
        assert float((got.float() - want).norm() / want.norm()) <= H


def test_results_repeat_and_a_captured_pass_replays(mp8):
    M, N, K = 300, 1100, 128
    c = case(14, M, N, K, ignored=0.1)
    x, w, t, loss, lse = forward(mp8, c)
    dx, dw = buffers(M, N, K, torch.float16)
    backward(mp8, c, x, w, t, loss, lse, scale=8.0, dx16=dx[:M * K], dw16=dw[:N * K])
    first = [v.clone() for v in (loss, lse, dx, dw)]
    ws = torch.empty(mp8.softmax_xent_bwd_workspace_bytes(M, N, K) + mp8.softmax_xent_fwd_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    g_loss, g_lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    gx, gw = buffers(M, N, K, torch.float16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, g_loss, g_lse, workspace=ws)
        mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, g_loss, g_lse, dx16=gx[:M * K], dw16=gw[:N * K], scale=8.0, workspace=ws)
    for _ in range(4):
        for v in (g_loss, g_lse, gx, gw):
            v.fill_(3.0)
        gx[M * K:], gw[N * K:] = 7.0, 7.0
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(first, (g_loss, g_lse, gx, gw)):
            assert torch.equal(a, b)


def test_two_calls_at_once_on_two_streams(mp8):
    M, N, K = 512, 900, 256
    cs = [case(20 + k, M, N, K) for k in range(2)]
    want = []
    for c in cs:
        x, w, t, loss, lse = forward(mp8, c)
        dx, dw = buffers(M, N, K, torch.float16)
        backward(mp8, c, x, w, t, loss, lse, dx16=dx[:M * K], dw16=dw[:N * K])
        want.append((x, w, t, loss.clone(), lse.clone(), dx, dw))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    got = [None, None]
    for _ in range(3):
        for k, s in enumerate(streams):
            x, w, t = want[k][:3]
            with torch.cuda.stream(s):
                loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
                ws = torch.empty(mp8.softmax_xent_bwd_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
                wf = torch.empty(mp8.softmax_xent_fwd_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
                dx, dw = buffers(M, N, K, torch.float16)
                mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=wf)
                mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dx16=dx[:M * K], dw16=dw[:N * K], workspace=ws)
                got[k] = (loss, lse, dx, dw, ws, wf)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for p, q in zip(a[3:], b[:4]):
            assert torch.equal(p, q)


def test_zero_dimensions_do_nothing(mp8):
    e16 = torch.empty(0, dtype=torch.float16, device="cuda")
    f = torch.full((4,), 5.0, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    mp8.softmax_xent_fwd_fp16(0, 8, 8, e16, torch.zeros(64, dtype=torch.float16, device="cuda"), none, f[:0], f[:0])
    mp8.softmax_xent_fwd_fp16(4, 0, 8, torch.zeros(32, dtype=torch.float16, device="cuda"), e16, t, f, f)
    torch.cuda.synchronize()
    assert bool((f == 5).all())
    assert mp8.softmax_xent_fwd_workspace_bytes(0, 8, 8) == mp8.softmax_xent_bwd_workspace_bytes(4, 0, 8) == 0
