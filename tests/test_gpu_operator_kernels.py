"""Every instance of the half-precision products, and of the kernel that makes the polynomial and multiplies by it, is launched by a call of the
tests that hold results to their definitions: the calls are recorded, not run, and their kernels' names are read."""
import itertools
import re

import pytest
import torch

import test_gpu_operator_rounding as rounding
import test_gpu_operator_tiles as tiles
import test_gpu_orthogonal_momentum as momentum
import test_gpu_softmax_xent as xent
from captured import launches
from test_gpu_operator_tiles import mp8  # noqa: F401

pytestmark = pytest.mark.gpu

TILES = {"256": (256, 256, 2, 1, 0), "192": (192, 192, 2, 1, 0), "128": (128, 128, 2, 2, 1), "64": (64, 64, 4, 2, 1), "64 by index": (64, 64, 8, 1, 2)}
PRODUCT = re.compile(r"half_gemm_kernelINS_10HalfTilingILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELNS_12HalfScheduleE(\d)EEELb(\d)ELb(\d)ENS_(\d+)(\w+)")
JOINT = re.compile(r"ortho_joint_kernelILi(\d)ELb(\d)ENS_(\d+)(\w+)")


def products(names):
    """(tile, operands that are contraction-major, epilogue and its option) of the products among them."""
    for name in names:
        if "half_gemm_kernel" not in name:
            continue
        m = PRODUCT.search(name)
        n, rest = int(m[8]), m[9]  # (a mangled name: its length, itself, its template's arguments)
        option = re.match(r"ILb(\d)E", rest[n:])
        yield (next(k for k, v in TILES.items() if v == tuple(map(int, m.groups()[:5]))), {"00": "", "01": "b", "11": "ab"}[m[6] + m[7]],
               rest[:n] + (option[1] if option else ""))


def empty(*shape, dtype=torch.uint8):
    return torch.empty(shape, dtype=dtype, device="cuda")


def cross_entropy(mp8, M, N, K):
    x, w, t = empty(M, K, dtype=torch.float16), empty(N, K, dtype=torch.float16), empty(M, dtype=torch.int64)
    loss, ws = empty(M, dtype=torch.float32), empty(max(mp8.softmax_xent_fwd_workspace_bytes(M, N, K), mp8.softmax_xent_bwd_workspace_bytes(M, N, K)))

    def call():
        mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, loss, workspace=ws)
        mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, loss, dx16=torch.empty_like(x), dw16=torch.empty_like(w), workspace=ws)
    return launches(call)


def update(mp8, batch, rows, cols):
    w, v, g = (empty(batch, rows, cols, dtype=d) for d in (torch.float16, torch.float32, torch.uint8))
    ws = empty(max(16, mp8.orthogonal_momentum_workspace_bytes(batch, rows, cols)))
    return launches(lambda: mp8.orthogonal_momentum_fp16_sr(w, v, g, 0.1, 1.0, 0.9, workspace=ws))


def test_every_product_of_the_cross_entropy(mp8):
    shapes = rounding.shapes_of(tiles.test_cross_entropy_of_large_tiles) + xent.SHAPES
    reached = set(itertools.chain.from_iterable(products(cross_entropy(mp8, *s)) for s in shapes))
    want = {(t, "", e) for t in TILES if t != "192" for e in ("XentStats", "XentError")}
    want |= {(t, o, e) for t in TILES for o in ("b", "ab") for e in ("HalfEpiSum", "XentOut0", "XentOut1")}
    assert reached == want, reached ^ want


def test_every_product_of_the_momentum(mp8):
    shapes = rounding.shapes_of(tiles.test_direction_of_large_tiles) + [(1, *s) for s in momentum.SHAPES]
    names = [n for s in shapes for n in update(mp8, *s)]
    reached = set(products(names))
    want = {(t, o, "OrthoSymmetric0") for t in TILES for o in ("", "ab")} | {(t, "", "OrthoSymmetric1") for t in TILES}
    want |= {(t, o, e + tall) for t in TILES for o, tall in (("b", "0"), ("", "1")) for e in ("OrthoNext", "OrthoUpdate")}
    assert reached == want, reached ^ want
    joint = {(int(m[1]), m[2], m[4][:int(m[3])]) for m in map(JOINT.search, names) if m}
    assert joint == set(itertools.product((1, 2, 3, 4), "01", ("OrthoNext", "OrthoUpdate"))), joint
