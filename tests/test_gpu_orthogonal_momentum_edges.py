"""GPU tests of mp8_orthogonal_momentum_fp16_sr over all numbers of steps, and for gradients of few directions."""
import math

import pytest
import torch

from test_gpu_operator_tiles import H, codes, iterate, momentum, mp8, values  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [12, 64])
@pytest.mark.parametrize("batch,rows,cols", [(1, 700, 333), (2, 1300, 421), (1, 2100, 1013), (1, 4999, 2049), (1, 333, 700), (1, 161, 93), (1, 1000, 7)])
def test_many_steps(mp8, steps, batch, rows, cols):
    """f(s) = 3.4445 s - 4.7750 s^3 + 2.0315 s^5 maps (0, 1.263] to (0, 1.2024] and [0.554, 1.2024] to [0.6816, 1.2024] (extrema at s^2 = 0.3075 and
    1.1028): from there singular values do not come out, however many steps follow, and those of noise get there within ten.  Every step's half
    operands are off by at most 2^-11 / sqrt 3 of their root mean square, independently, which moves a singular value by at most (sqrt m + sqrt n) / sqrt n
    <= 2 times that, times a gain of at most |a| + 4 |b| + 6 |c| < 35: 0.02."""
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    g = codes(torch.randn((batch, rows, cols), generator=gen, device="cuda"))
    v, w = torch.zeros(g.shape, device="cuda"), torch.zeros(g.shape, dtype=torch.float16, device="cuda")
    momentum(mp8, w, v, g, -1.0, nesterov=False, steps=steps)
    assert bool(torch.isfinite(w).all())
    for i in {0, batch - 1}:
        s = torch.linalg.svdvals(w[i].double())
        assert float(s.max()) <= 1.2024 + 0.02
        # (a square matrix of noise has singular values near zero, which take longer)
        if max(rows, cols) >= 1.5 * min(rows, cols):
            assert float(s.min()) >= 0.6816 - 0.02


# what the header says X may be off by, of its root mean square, where k directions hold most of u; noise in units of their size
STATED = {0.2: lambda k: 4e-3, 0.05: lambda k: 7e-3, 0.01: lambda k: 2.5e-2, 0.0: lambda k: 0.17 / math.sqrt(k)}


@pytest.mark.parametrize("noise", STATED)
@pytest.mark.parametrize("k", [1, 2, 8, 32])
@pytest.mark.parametrize("rows,cols", [(64, 256), (256, 256), (128, 1152), (1024, 1024), (1000, 300), (100, 8000)])
def test_few_directions(mp8, rows, cols, k, noise):
    """A first rounding to half leaves errors in all directions, which grow by a = 3.4445 per step, as the definition has it: 0.29 * 2^-11 of the norm
    of u becomes some 0.14, beside k directions of about 1.  The kernel is as far from the exact iteration as the model of its roundings is
    (twice that and a rounding of the result is asserted), and as the header says."""
    gen = torch.Generator(device="cuda").manual_seed(rows + k)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda")
    v = noise * draw(rows, cols) + draw(rows, k) @ draw(k, cols) / math.sqrt(k)
    g, w = torch.zeros((rows, cols), dtype=torch.uint8, device="cuda"), torch.zeros((rows, cols), dtype=torch.float16, device="cuda")
    u = v.double()
    ws = torch.empty(mp8.orthogonal_momentum_workspace_bytes(1, rows, cols), dtype=torch.uint8, device="cuda")
    mp8.orthogonal_momentum_fp16_sr(w, v, g, -1.0, 1.0, 1.0, nesterov=False, round=mp8.RNE, workspace=ws)
    exact, model = iterate(u, 5, False), iterate(u, 5, True, diagonal=False)
    off, norm = float((w.double() - exact).norm()), float(exact.norm())
    assert off <= 2 * float((model - exact).norm()) + H * norm
    assert off <= STATED[noise](k) * norm
