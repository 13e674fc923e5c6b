"""GPU tests of the softmax cross entropy and the orthogonalised momentum at sizes that fill the larger tiles, cut contractions and the
vocabulary into pieces and leave odd edges, against their definitions in 64 bits (on the GPU, in torch), and of a training step in which
both are used together with the 8-bit layers.  Tolerances as derived in test_gpu_softmax_xent.py and test_gpu_orthogonal_momentum.py."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U, H = 2.0 ** -24, 2.0 ** -11
A, B, C = 3.4445, -4.7750, 2.0315


@pytest.fixture(scope="module")
def mp8():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1905_12334_amd as m
    m.lib()
    return m


def codes(x):
    return x.float().to(torch.float8_e5m2).view(torch.uint8)


def values(c):
    return c.view(torch.float8_e5m2).double()


def bytes_of(n):
    return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------ softmax cross entropy
def truth(x, w, t, scale):
    """Results in 64 bits and the elementwise bounds; scale: of all tokens, or of each."""
    scale = torch.as_tensor(scale, dtype=torch.float64, device="cuda").expand(x.shape[0])
    (M, K), N = x.shape, w.shape[0]
    live = (t >= 0) & (t < N)
    at, rows = torch.where(live, t, 0), torch.arange(M, device="cuda")
    z = x @ w.t()
    dz = K * U * (x.abs() @ w.abs().t()).amax(1)
    lse = torch.logsumexp(z, 1)
    spread = (z.amax(1) - z.amin(1)) / math.log(2) + 1
    r = 2 * dz + (math.log(2) * spread + 64 + N / 32 + 16) * U
    others = torch.exp(z - z[rows, at][:, None])
    others[rows, at] = 0
    loss = torch.where(live, torch.log1p(others.sum(1)), 0.0)
    del others
    e = torch.exp(z - lse[:, None])
    e[rows[live], t[live]] = torch.expm1(-loss[live])
    e = torch.where(live[:, None], e, 0.0) * scale[:, None]
    dlse = r + 4 * U * lse.abs()  # (of tokens without a target too)
    r = torch.where(live, r, 0.0)
    de = (H + r + 8 * U)[:, None] * e.abs() + torch.where(live, 2.0 ** -39 * scale[live].abs().max(), 0.0)[:, None]
    dx, dw = e @ w, e.t() @ x
    bx, bw = de @ w.abs() + N * U * (e.abs() @ w.abs()), de.t() @ x.abs() + M * U * (e.abs().t() @ x.abs())
    return dict(loss=loss, lse=lse, r=r, dlse=dlse, dx=dx, dw=dw, bx=bx, bw=bw, live=live)


def inputs(seed, M, N, K):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = (torch.randn((N, K), generator=gen, device="cuda") * K ** -0.5).half()
    t = torch.randint(0, N, (M,), generator=gen, device="cuda")
    x = (torch.randn((M, K), generator=gen, device="cuda") + 4 * torch.rand((M, 1), generator=gen, device="cuda") * w[t].float()).half()
    t[torch.rand(M, generator=gen, device="cuda") < 0.1] = -100
    return x, w, t


def within(got, want, bound, what):
    off = (got.double().view_as(want) - want).abs()
    assert bool((off <= bound).all()), (what, float((off / bound).max()))


@pytest.mark.parametrize("M,N,K", [(2055, 4099, 136), (3001, 9001, 72), (4099, 8200, 520), (1111, 40009, 264), (9001, 1999, 1032), (512, 20001, 2056),
                                   (8200, 40001, 40), (921, 16507, 386), (893, 18915, 472), (1, 34847, 136), (1, 36418, 135), (1215, 14131, 16),
                                   (22139, 2, 2032), (15981, 937, 16), (33505, 2, 8), (37658, 2, 144), (34686, 756, 256), (1, 76922, 1), (35368, 2, 1),
                                   (21873, 2, 324), (33885, 858, 194), (8709, 31376, 1), (1, 33607, 1), (10116, 5634, 134), (19893, 395, 4304),
                                   (15724, 6555, 1), (9620, 9091, 400), (2500, 20003, 1999)])
def test_cross_entropy_of_large_tiles(mp8, M, N, K):
    x, w, t = inputs(M + N, M, N, K)
    scale = 256.0 / M
    want = truth(x.double(), w.double(), t, scale)
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=bytes_of(mp8.softmax_xent_fwd_workspace_bytes(M, N, K)))
    within(lse, want["lse"], want["dlse"], "lse")
    within(loss, want["loss"], want["loss"] * (want["r"] + 4 * U) + 1e-44, "loss")
    ws = bytes_of(mp8.softmax_xent_bwd_workspace_bytes(M, N, K))
    dx, dw = torch.full((M * K + 64,), 7.0, dtype=torch.float16, device="cuda"), torch.full((N * K + 64,), 7.0, dtype=torch.float16, device="cuda")
    sx, sw = mp8.new_stats(), mp8.new_stats()
    mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dx16=dx[:M * K], dw16=dw[:N * K], scale=scale, dx_stats=sx, dw_stats=sw, workspace=ws)
    assert bool((dx[M * K:] == 7).all()) and bool((dw[N * K:] == 7).all())
    for got, key, n, stats in ((dx, "x", M * K, sx), (dw, "w", N * K, sw)):
        value, bound = want["d" + key], want["b" + key]
        within(got[:n], value, bound + H * (value.abs() + bound) + 2.0 ** -25, "d" + key)
        if M > 50 and N > 50:  # (many roundings in a sum, many sums)
            assert float((got[:n].double().view_as(value) - value).norm() / value.norm()) <= H
        amax, bad, _ = mp8.read_stats(stats)
        top = torch.tensor([amax], dtype=torch.int32).view(torch.float32)
        assert bad == 0 and abs(float(top) - float(value.abs().max())) <= float(bound.max())
    # codes, alone and beside the halves, which stay the same
    for sr in (False, True):
        cx, cw = torch.full((M * K + 64,), 0xAA, dtype=torch.uint8, device="cuda"), torch.full((N * K + 64,), 0xAA, dtype=torch.uint8, device="cuda")
        ax, aw = torch.empty_like(x), torch.empty_like(w)
        kw = dict(scale=scale, round=mp8.SR if sr else mp8.RNE, seed=5, dx_offset=1, dw_offset=2)
        mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dx8=cx[:M * K], dw8=cw[:N * K], dx16=ax, dw16=aw, workspace=ws, **kw)
        assert torch.equal(ax.view(-1), dx[:M * K]) and torch.equal(aw.view(-1), dw[:N * K])
        assert bool((cx[M * K:] == 0xAA).all()) and bool((cw[N * K:] == 0xAA).all())
        for got, key, n in ((cx, "x", M * K), (cw, "w", N * K)):
            # a step of a value is 2^-2 of its power of two; subnormal steps are 2^-16
            value, bound = want["d" + key], want["b" + key]
            step = torch.maximum(torch.exp2(torch.floor(torch.log2(value.abs() + bound))) / 4, torch.tensor(2.0 ** -16, device="cuda"))
            within(values(got[:n]), value, bound + step * (1.0 if sr else 0.5), "code of d" + key)
        only = torch.empty(N * K, dtype=torch.uint8, device="cuda")
        mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dw8=only, workspace=ws, **kw)
        assert torch.equal(only, cw[:N * K])
        only = torch.empty(M * K, dtype=torch.uint8, device="cuda")
        mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dx8=only, workspace=ws, **kw)
        assert torch.equal(only, cx[:M * K])


@pytest.mark.parametrize("size", [1e-42, 1e-37, 1e37, 3e38])
def test_token_weights_to_the_ends_of_fp32(mp8, size):
    M, N, K = 200, 300, 64
    x, w, t = inputs(5, M, N, K)
    weight = torch.full((M,), size, device="cuda")
    weight[::3] *= 0.25
    # (what FP32 makes of the weights; the scale's FP32 rounding is one of the 8 U in the bound)
    scale = torch.tensor(min(16 / size, 2.0 ** 126), dtype=torch.float32).item()
    want = truth(x.double(), w.double(), t, (weight.double() * scale))
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=bytes_of(mp8.softmax_xent_fwd_workspace_bytes(M, N, K)))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dloss=weight, dx16=dx, dw16=dw, scale=scale,
                              workspace=bytes_of(mp8.softmax_xent_bwd_workspace_bytes(M, N, K)))
    for got, key in ((dx, "x"), (dw, "w")):
        value, bound = want["d" + key], want["b" + key]
        within(got, value, bound + H * (value.abs() + bound) + 2.0 ** -25, "d" + key)


# ------------------------------------------------------------------ orthogonalised momentum
def iterate(u, steps, rounded, diagonal=True):
    """X after `steps`; `rounded`: with the operands rounded to half as stored (X times s, A and the polynomial times 2^14), the polynomial's
    diagonal too or not."""
    tall = u.shape[0] > u.shape[1]
    u = u.t().contiguous() if tall else u
    x = u / u.norm()
    s = 2.0 ** round(0.5 * math.log2(u.shape[1]))
    half = (lambda v, f: (v * f).half().double() / f) if rounded else (lambda v, f: v)
    x = half(x, s)
    for k in range(steps):
        a = half(x @ x.t().contiguous(), 2.0 ** 14)
        p = B * a + C * (a @ a)
        p = half(p, 2.0 ** 14) if diagonal else half(p, 2.0 ** 14).fill_diagonal_(0.0) + torch.diag(p.diagonal())
        x = A * x + p @ x
        if k + 1 < steps:
            x = half(x, s)
    return x.t().contiguous() if tall else x


def momentum(mp8, w, v, g, lr, **kw):
    batch = w.numel() // (w.shape[-1] * w.shape[-2])
    ws = bytes_of(mp8.orthogonal_momentum_workspace_bytes(batch, *w.shape[-2:]))
    mp8.orthogonal_momentum_fp16_sr(w, v, g, lr, 1.0, 0.9, round=mp8.RNE, workspace=ws, **kw)


@pytest.mark.parametrize("batch,rows,cols", [
    (1, 40, 8192), (1, 8192, 40), (5, 30, 2100), (3, 3001, 65), (2, 100, 5000), (1, 1, 20000), (1, 129, 30001), (1, 260, 8192), (1, 1024, 1024),
    (1, 1001, 1003), (9, 500, 520), (20, 257, 389), (1, 1500, 1499), (1, 2049, 2560), (2, 2100, 4099), (1, 4100, 3700), (1, 700, 20011), (1, 20011, 700),
    (1, 4104, 6200), (61, 3571, 1), (54, 886, 1), (37, 303, 269), (3, 1631, 1170), (35, 597, 564), (4, 5039, 1281), (15, 1244, 972), (1, 15047, 2989),
    (54, 2, 896), (21, 1, 10872), (43, 259, 283), (3, 1128, 1413), (41, 575, 712), (8, 920, 5333), (16, 1001, 1032), (1, 2956, 13518), (1, 835, 901),
    (1, 854, 835), (13, 2732, 134), (16, 132, 2134), (1, 865, 9807), (1, 8478, 994),
    (1, 64, 64), (70, 64, 1000), (70, 1000, 64), (1, 127, 129), (1, 129, 127), (6, 128, 700), (6, 700, 128), (9, 128, 4000), (2, 160, 1000), (2, 1000, 185),
    (1, 192, 192), (1, 193, 255), (3, 256, 256), (1, 3000, 249), (1, 250, 9000), (1, 2313, 2016), (13, 6244, 519),
    (5, 846, 2519)])
def test_direction_of_large_tiles(mp8, batch, rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    g = codes(torch.randn((batch, rows, cols), generator=gen, device="cuda"))
    v = torch.zeros((batch, rows, cols), device="cuda")
    n = batch * rows * cols
    w = torch.zeros(n + 64, dtype=torch.float16, device="cuda")
    w[n:] = 7
    momentum(mp8, w[:n].view(batch, rows, cols), v, g, -1.0, nesterov=False)
    assert torch.equal(v.double(), values(g)) and bool((w[n:] == 7).all())
    got = w[:n].view(batch, rows, cols)
    for i in {0, batch - 1}:
        u = v[i].double()
        exact, model = iterate(u, 5, False), iterate(u, 5, True)
        assert float((got[i].double() - exact).norm()) <= float(2 * (model - exact).norm() + H * exact.norm())
    # again, the same bits: what is added in several parts is added in their order
    again, v2 = torch.zeros_like(got), torch.zeros_like(v)
    momentum(mp8, again, v2, g, -1.0, nesterov=False)
    assert torch.equal(again, got)


@pytest.mark.parametrize("rows,cols", [(60, 4000), (1152, 128), (200, 300), (700, 1500), (2001, 1013), (2050, 3000)])
def test_the_polynomials_diagonal_is_not_rounded(mp8, rows, cols):
    """The direction of noise is about as far from the exact iteration as the model whose polynomial keeps its diagonal, which is far better
    than the other one; the result's own rounding (H / sqrt 3 of the norm, independent) comes on top.  Sums of thousands of roundings: 10 %."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    g = codes(torch.randn((rows, cols), generator=gen, device="cuda"))
    v, w = torch.zeros((rows, cols), device="cuda"), torch.zeros((rows, cols), dtype=torch.float16, device="cuda")
    momentum(mp8, w, v, g, -1.0, nesterov=False)
    u = v.double()
    exact, kept, lost = iterate(u, 5, False), iterate(u, 5, True, diagonal=False), iterate(u, 5, True)
    kept, lost, own = float((kept - exact).norm()), float((lost - exact).norm()), H / math.sqrt(3) * float(exact.norm())
    assert kept < 0.85 * lost
    assert float((w.double() - exact).norm()) <= 1.1 * math.hypot(kept, own)


def test_two_momentum_calls_at_once_on_two_streams(mp8):
    shapes = [(1, 128, 6000), (4, 300, 400)]
    gen = torch.Generator(device="cuda").manual_seed(1)
    data = [(torch.randn(s, generator=gen, device="cuda"), codes(torch.randn(s, generator=gen, device="cuda"))) for s in shapes]
    want = []
    for v, g in data:
        w = torch.zeros(v.shape, dtype=torch.float16, device="cuda")
        v = v.clone()
        momentum(mp8, w, v, g, -1.0)
        want.append((w, v))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in shapes]
    for _ in range(3):
        got = []
        for (v, g), s in zip(data, streams):
            with torch.cuda.stream(s):
                w, v = torch.zeros(v.shape, dtype=torch.float16, device="cuda"), v.clone()
                momentum(mp8, w, v, g, -1.0)
                got.append((w, v))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------ large offsets, shared workspaces
def test_cross_entropy_beyond_2_to_the_31_elements(mp8):
    M, N, K = 1 << 22, 67, 520
    x, w, t = inputs(3, M, N, K)
    assert x.numel() > 1 << 31
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=torch.empty(mp8.softmax_xent_fwd_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda"))
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    scale = 256.0 / M
    mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dx16=dx, dw16=dw, scale=scale,
                              workspace=torch.empty(mp8.softmax_xent_bwd_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda"))
    dw_want, bw = torch.zeros((N, K), dtype=torch.float64, device="cuda"), torch.zeros((N, K), dtype=torch.float64, device="cuda")
    part = 1 << 19
    for i in range(0, M, part):
        rows = slice(i, i + part)
        want = truth(x[rows].double(), w.double(), t[rows], scale)
        within(loss[rows], want["loss"], want["loss"] * (want["r"] + 4 * U) + 1e-44, "loss")
        within(dx[rows], want["dx"], want["bx"] + H * (want["dx"].abs() + want["bx"]) + 2.0 ** -25, "dx")
        dw_want += want["dw"]
        bw += want["bw"]
    # (additions of the parts: M U of all terms covers them, their own bound has part U)
    within(dw, dw_want, bw * (M // part) + H * (dw_want.abs() + bw) + 2.0 ** -25, "dw")
    assert float((dw.double() - dw_want).norm() / dw_want.norm()) <= H


def test_momentum_beyond_2_to_the_31_elements(mp8):
    batch, rows, cols = 65535, 64, 520
    gen = torch.Generator(device="cuda").manual_seed(4)
    few = codes(torch.randn((101, rows, cols), generator=gen, device="cuda"))
    g = torch.empty((batch, rows, cols), dtype=torch.uint8, device="cuda")
    for i in range(0, batch, 101):
        g[i:i + 101] = few[:min(101, batch - i)]
    assert g.numel() > 1 << 31
    v = torch.zeros(g.shape, device="cuda")
    w = torch.zeros(g.shape, dtype=torch.float16, device="cuda")
    ws = torch.empty(mp8.orthogonal_momentum_workspace_bytes(batch, rows, cols), dtype=torch.uint8, device="cuda")
    mp8.orthogonal_momentum_fp16_sr(w, v, g, -1.0, 1.0, 0.9, nesterov=False, round=mp8.RNE, workspace=ws)
    for i in range(0, batch, 101):  # the same matrix, the same direction, wherever it lies
        n = min(101, batch - i)
        assert torch.equal(w[i:i + n], w[:n]) and torch.equal(v[i:i + n], v[:n])
    for i in (0, 100):
        u = values(few[i])
        exact, model = iterate(u, 5, False), iterate(u, 5, True)
        assert float((w[i].double() - exact).norm()) <= float(2 * (model - exact).norm() + H * exact.norm())


def test_captured_graphs_that_share_a_workspace(mp8):
    gen = torch.Generator(device="cuda").manual_seed(9)
    shapes = [(1, 128, 6000), (2, 200, 300), (1, 40, 9000)]  # (sliced products, whose counters lie in the workspace, and others)
    M, N, K = 300, 2000, 200
    x, t_w, t = inputs(2, M, N, K)
    need = [mp8.orthogonal_momentum_workspace_bytes(*s) for s in shapes] + [mp8.softmax_xent_fwd_workspace_bytes(M, N, K), mp8.softmax_xent_bwd_workspace_bytes(M, N, K)]
    ws = bytes_of(max(need))
    data = [(codes(torch.randn(s, generator=gen, device="cuda")), torch.zeros(s, dtype=torch.float16, device="cuda"), torch.zeros(s, device="cuda")) for s in shapes]
    out = [torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty_like(x), torch.empty_like(t_w)]

    def update(g, w, v):
        mp8.orthogonal_momentum_fp16_sr(w, v, g, 0.1, 1.0, 0.9, seed=2, offset=3, workspace=ws)

    def loss(a, b, dx, dw):
        mp8.softmax_xent_fwd_fp16(M, N, K, x, t_w, t, a, b, workspace=ws)
        mp8.softmax_xent_bwd_fp16(M, N, K, x, t_w, t, a, b, dx16=dx, dw16=dw, workspace=ws)
    eager = [(g, w.clone(), v.clone()) for g, w, v in data]
    eager_out = [a.clone() for a in out]
    graphs = []
    for call, args in [(update, d) for d in data] + [(loss, out)]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(*args)
        graphs.append(graph)
    for k in range(4):
        for j in ((0, 1, 2, 3), (3, 2, 1, 0), (1, 3, 0, 2), (2, 0, 3, 1))[k]:
            graphs[j].replay()
        torch.cuda.synchronize()
        for d in eager:
            update(*d)
        loss(*eager_out)
        torch.cuda.synchronize()
        for a, b in zip(data, eager):
            assert torch.equal(a[1], b[1]) and torch.equal(a[2], b[2])
        for a, b in zip(out, eager_out):
            assert torch.equal(a, b)


# ------------------------------------------------------------------ together
class Step:
    """A training step: an 8-bit layer, ReLU on the codes, a last layer in FP16 with the cross entropy, the layer's weights by
    orthogonalised momentum, the last layer's by plain momentum, both left out where a gradient overflowed."""

    def __init__(self, mp8, M=1008, D=264, K=520, N=3001):
        self.mp8, self.M, self.D, self.K, self.N = mp8, M, D, K, N
        gen = torch.Generator(device="cuda").manual_seed(7)
        u8, dev = torch.uint8, "cuda"
        empty = lambda *s, d=u8: torch.empty(s, dtype=d, device=dev)
        self.x8 = codes(torch.randn((M, D), generator=gen, device=dev))
        self.t = torch.randint(0, N, (M,), generator=gen, device=dev)
        self.t[::17] = -100
        self.w1 = (torch.randn((K, D), generator=gen, device=dev) * (2 / D) ** 0.5).half()
        self.w2 = (torch.randn((N, K), generator=gen, device=dev) * K ** -0.5).half()
        self.w1_8 = codes(self.w1)
        self.v1, self.v2 = torch.zeros((K, D), device=dev), torch.zeros((N, K), device=dev)
        self.h8, self.r8, self.dr8, self.dh8, self.g1, self.g2 = empty(M, K), empty(M, K), empty(M, K), empty(M, K), empty(K, D), empty(N, K)
        self.loss, self.lse = empty(M, d=torch.float32), empty(M, d=torch.float32)
        self.stats = mp8.new_stats()
        need = max(mp8.softmax_xent_fwd_workspace_bytes(M, N, K), mp8.softmax_xent_bwd_workspace_bytes(M, N, K),
                   mp8.orthogonal_momentum_workspace_bytes(1, K, D), 64 << 20)
        self.ws = empty(need)

    def state(self):
        return [a.clone() for a in (self.w1, self.w2, self.w1_8, self.v1, self.v2, self.loss, self.g1, self.g2)]

    def run(self, loss_scale, lr=0.02):
        m, M, D, K, N = self.mp8, self.M, self.D, self.K, self.N
        scale = loss_scale / M
        m.gemm_fp8(m.FWD, M, K, D, self.x8, self.w1_8, out8=self.h8, workspace=self.ws)
        torch.mul(self.h8, self.h8 < 0x80, out=self.r8)
        m.softmax_xent_fwd_fp16(M, N, K, self.r8, self.w2, self.t, self.loss, self.lse, workspace=self.ws)
        self.stats.zero_()
        m.softmax_xent_bwd_fp16(M, N, K, self.r8, self.w2, self.t, self.loss, self.lse, dx8=self.dr8, dw8=self.g2, scale=scale,
                                dx_stats=self.stats, dw_stats=self.stats, workspace=self.ws)
        torch.mul(self.dr8, self.r8 != 0, out=self.dh8)
        m.gemm_fp8(m.WGRAD, M, D, K, self.dh8, self.x8, out8=self.g1, stats=self.stats, workspace=self.ws, flags=m.FLAG_CONTRACTION_MAJOR)
        bad = self.stats.view(torch.int32)[1:2]
        m.orthogonal_momentum_fp16_sr(self.w1, self.v1, self.g1, lr, 1.0 / loss_scale, 0.9, seed=3, offset=1, skip_if_nonzero=bad, w8_out=self.w1_8,
                                      workspace=self.ws)
        m.sgd_momentum_fp16_sr(self.w2, self.v2, self.g2, lr, 1.0 / loss_scale, 0.9, seed=3, offset=2, skip_if_nonzero=bad)


def half_step(v):
    """Half a step of the 8-bit format at |v|: 2^-3 of it at most, 2^-17 below the smallest normal value."""
    return 2.0 ** -3 * v.abs() + 2.0 ** -17


def test_a_training_step_with_both(mp8):
    s = Step(mp8)
    w1, w2, loss_scale, lr = s.w1.clone(), s.w2.clone(), 256.0, 0.02
    s.run(loss_scale, lr)
    want = truth(values(s.r8), w2.double(), s.t, loss_scale / s.M)
    within(s.loss, want["loss"], want["loss"] * (want["r"] + 4 * U) + 1e-44, "loss")
    within(values(s.dr8), want["dx"], want["bx"] + half_step(want["dx"].abs() + want["bx"]), "dx")
    within(values(s.g2), want["dw"], want["bw"] + half_step(want["dw"].abs() + want["bw"]), "dw")
    # through the first layer: what the codes of dx may be off by, the product's FP32 sums, one rounding
    on, x = (s.r8 != 0).double(), values(s.x8)
    dx, off = want["dx"] * on, (want["bx"] + half_step(want["dx"].abs() + want["bx"])) * on
    g = dx.t() @ x
    bound = off.t() @ x.abs() + s.M * U * ((dx.abs() + off).t() @ x.abs())
    within(values(s.g1), g, bound + half_step(g.abs() + bound), "gradient of the first layer")
    # the first layer's update: direction, stochastic rounding (less than a step, 2^-10), the 8-bit copy
    assert torch.equal(s.v1.double(), values(s.g1) / loss_scale)
    u = values(s.g1) * 1.9 / loss_scale
    exact, model = iterate(u, 5, False), iterate(u, 5, True)
    new = w1.double() - lr * exact
    slack = lr * (2 * (model - exact).norm() + H * exact.norm()) + 2.0 ** -10 * new.norm()
    assert float((s.w1.double() - new).norm()) <= float(slack)
    assert torch.equal(s.w1_8, codes(s.w1)) and not torch.equal(s.w2, w2)


def test_captured_training_steps_and_one_that_overflows(mp8):
    eager, captured = Step(mp8), Step(mp8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run(256.0)
    for _ in range(4):
        captured.ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        eager.ws.fill_(0xAA)
        eager.run(256.0)
        torch.cuda.synchronize()
        for a, b in zip(captured.state(), eager.state()):
            assert torch.equal(a, b)
        assert mp8.read_stats(eager.stats)[1] == 0
    before = eager.state()
    eager.run(2.0 ** 40)
    assert mp8.read_stats(eager.stats)[1] > 0
    for a, b in zip(before[:5], eager.state()):
        assert torch.equal(a, b)
