"""GPU tests of what the softmax cross entropy and the orthogonalised momentum round stochastically, and of the zeros that they count, in every
tile and with every pass that adds up slices or pieces: with the bits that the element's own index has in the stream (mp8_sr_bits, which
other tests hold to the oracle).  What is rounded is known from the same call's result as a half to nearest, which other tests hold to the
definition: to within 2^-11 of it and 2^-25.  Rounding is monotone for an element's bits, so the result lies between what the two ends
become: one value for most elements.  The check is shown to notice another element's bits by giving them to the oracle."""
import numpy as np
import pytest
import torch

import test_gpu_operator_tiles as tiles
from test_gpu_operator_tiles import H, U, bytes_of, codes, inputs, mp8, truth, values  # noqa: F401

pytestmark = pytest.mark.gpu
SEED = 0x1234567890


def shapes_of(test):
    return next(m.args[1] for m in test.pytestmark if m.name == "parametrize")


def bits(mp8, n, offset):
    out = torch.empty(n, dtype=torch.int16, device="cuda")
    mp8.sr_bits(out, SEED, offset)
    return out.double() % 65536


def stochastic(v, r, fraction):
    """Finite values of the format with exponents of 5 bits: the magnitude in units of 2^-16 of a step, r added, whole steps."""
    step = torch.exp2((torch.frexp(v.abs())[1] - 1).clamp(min=-14).double() - fraction)
    return torch.copysign(torch.floor((torch.floor(v.abs() / step * 65536) + r) / 65536) * step, v)


def check_bits(mp8, got, value, slack, offset, fraction, what):
    """got, the rounding of something within slack of value."""
    got, value, slack = got.reshape(-1).double(), value.reshape(-1), slack.reshape(-1)
    r = bits(mp8, got.numel(), offset)
    inside = lambda r: (stochastic(value - slack, r, fraction) <= got) & (got <= stochastic(value + slack, r, fraction))
    assert bool(inside(r).all()), (what, int((~inside(r)).sum()))
    if got.numel() > 2000:
        assert float((~inside(torch.roll(r, 1))).double().mean()) > 0.02, what


def check_zeros(mp8, stats, got, value, bound, nonzero, what):
    """got, where `nonzero` surely was not rounded from a zero."""
    zero, n = got.reshape(-1) == 0, mp8.read_stats(stats)[2]
    surely = int((zero & nonzero).sum())
    assert surely <= n <= int((zero & (value.abs() + bound > 0)).sum()), (what, n)
    return surely


def passes(mp8, M, N, K, x, w, t):
    """A call of the backward pass with buffers of its own, and the forward pass's results."""
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=bytes_of(mp8.softmax_xent_fwd_workspace_bytes(M, N, K)))
    ws = bytes_of(mp8.softmax_xent_bwd_workspace_bytes(M, N, K))
    return lambda **kw: mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, workspace=ws, **kw)


def check_gradients(mp8, M, N, K, x, w, t, want, backward, scale):
    for key, n, offset in (("x", M * K, 5), ("w", N * K, 6)):
        value, bound = want["d" + key].reshape(-1), want["b" + key].reshape(-1)
        out, half = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.float16, device="cuda")
        backward(scale=scale, **{f"d{key}16": half})
        tiles.within(half, value, bound + H * (value.abs() + bound) + 2.0 ** -25, "d" + key)
        backward(scale=scale, round=mp8.SR, seed=SEED, **{f"d{key}8": out, f"d{key}_offset": offset})
        half = half.double()
        check_bits(mp8, values(out), half, 1.001 * H * half.abs() + 2.0 ** -25, offset, 2, "d" + key)
        # about half of the values below half the smallest step, at a scale for that: a power of two times the sums that are no zeros above
        size = float(value[value != 0].abs().median())
        for smallest, dtype, arg in ((2.0 ** -16, torch.uint8, "8"), (2.0 ** -24, torch.float16, "16")):
            f = 2.0 ** round(np.log2(smallest / 2 / size))
            out, stats = torch.empty(n, dtype=dtype, device="cuda"), mp8.new_stats()
            backward(scale=scale * f, **{f"d{key}{arg}": out, f"d{key}_stats": stats})
            got = values(out) if dtype == torch.uint8 else out
            flushed = check_zeros(mp8, stats, got, value * f, bound * f, half != 0, f"zeros of d{key}{arg}")
            assert flushed > 0 or n < 2000


@pytest.mark.parametrize("M,N,K", [s for s in shapes_of(tiles.test_cross_entropy_of_large_tiles)] + [(50, 77, 37), (130, 200, 96), (256, 1000, 2048)])
def test_gradients_of_every_tile(mp8, M, N, K):
    x, w, t = inputs(M + N, M, N, K)
    if M == 1:
        t[0] = N // 2
    scale = 256.0 / M
    want = truth(x.double(), w.double(), t, scale)
    check_gradients(mp8, M, N, K, x, w, t, want, passes(mp8, M, N, K, x, w, t), scale)


@pytest.mark.parametrize("M,N,K", [(40000, 9000, 64), (40001, 9001, 65), (64, 40000, 4096), (65, 40001, 4100), (90, 41000, 4101)])
def test_gradients_of_several_pieces(mp8, M, N, K):
    """More classes than one piece of the backward pass holds: rows of dw behind the first piece have their own indices too, whether a tile stores
    them or the pass that adds up slices."""
    assert (N - 1) * max(2 * M, 4 * -(-K // 64) * 64) > 512 << 20
    x, w, t = inputs(M + N, M, N, K)
    scale = 256.0 / M
    want = truth(x.double(), w.double(), t, scale)
    check_gradients(mp8, M, N, K, x, w, t, want, passes(mp8, M, N, K, x, w, t), scale)


@pytest.mark.parametrize("batch,rows,cols", [s for s in shapes_of(tiles.test_direction_of_large_tiles)] + [(4, 300, 400), (3, 640, 895), (24, 512, 512)])
def test_weights_of_every_tile(mp8, batch, rows, cols):
    """w' is half(fma(-lr, fma(wd, w, X), w)): with X as a call on zero weights leaves it, exact to a half's rounding."""
    n = batch * rows * cols
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    g = codes(torch.randn((batch, rows, cols), generator=gen, device="cuda"))
    zeros = lambda d: torch.zeros((batch, rows, cols), dtype=d, device="cuda")
    x = zeros(torch.float16)
    tiles.momentum(mp8, x, zeros(torch.float32), g, -1.0)
    w = (torch.randn((batch, rows, cols), generator=gen, device="cuda") * 0.05).half()
    lr, wd = float(np.float32(0.03)), float(np.float32(0.1))
    got, w8 = w.clone(), torch.full((n + 64,), 0xAA, dtype=torch.uint8, device="cuda")
    mp8.orthogonal_momentum_fp16_sr(got, zeros(torch.float32), g, lr, 1.0, 0.9, weight_decay=wd, round=mp8.SR, seed=SEED, offset=9, w8_out=w8[:n],
                                    workspace=bytes_of(mp8.orthogonal_momentum_workspace_bytes(batch, rows, cols)))
    x, wide = x.double(), w.double()
    new = wide - lr * (x + wd * wide)
    slack = lr * (H * x.abs() + 2.0 ** -25) + 4 * U * wide.abs()
    check_bits(mp8, got, new, slack, 9, 10, "weights")
    assert torch.equal(w8[:n], codes(got).reshape(-1)) and bool((w8[n:] == 0xAA).all())
