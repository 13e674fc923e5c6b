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
