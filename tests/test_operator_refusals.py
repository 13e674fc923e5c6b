"""What the softmax cross entropy and the orthogonalised momentum refuse, before anything is enqueued: no GPU is needed."""
import ctypes as C

import pytest
import torch

import paper_1905_12334_amd as mp8

OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, 1, 2, 3, 4
P = C.c_void_p(4096)       # an aligned address that is never followed
ODD = C.c_void_p(4096 + 8)
BIG = 1 << 40


def fwd(M=4, N=8, K=8, x=P, codes=0, ldx=8, w=P, ldw=8, t=P, loss=P, lse=P, ws=P, n=BIG):
    return mp8.lib().mp8_softmax_xent_fwd_fp16(M, N, K, x, codes, ldx, w, ldw, t, loss, lse, ws, n, None)


def bwd(M=4, N=8, K=8, x=P, codes=0, ldx=8, w=P, ldw=8, t=P, loss=P, lse=P, dloss=None, dx16=P, dx8=None, dw16=None, dw8=None,
        round=0, flags=0, ws=P, n=BIG):
    return mp8.lib().mp8_softmax_xent_bwd_fp16(M, N, K, x, codes, ldx, w, ldw, t, loss, lse, dloss, 1.0, dx16, dx8, dw16, dw8, round, flags,
                                               0, 0, 0, None, None, ws, n, None)


def ortho(batch=1, rows=8, cols=8, w=P, v=P, g=P, steps=5, round=1, skip=None, w8=None, stats=None, ws=P, n=BIG):
    return mp8.lib().mp8_orthogonal_momentum_fp16_sr(batch, rows, cols, w, v, g, 0.1, 1.0, 0.9, 1, 0.0, steps, round, 0, 0, skip, w8,
                                                     stats, ws, n, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_cross_entropy_refuses(call):
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(ldx=7), dict(ldw=7), dict(x=None), dict(w=None), dict(t=None), dict(loss=None),
                dict(lse=None)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(M=(1 << 22) + 1), dict(N=(1 << 22) + 1), dict(K=(1 << 20) + 1, ldx=1 << 21, ldw=1 << 21), dict(ldx=(1 << 21) + 1),
                dict(ldw=1 << 62), dict(M=1 << 22, N=1 << 22), dict(M=2 ** 62)):
        assert call(**bad) == UNSUPPORTED, bad
    for bad in (dict(x=ODD), dict(w=ODD), dict(ws=ODD)):
        assert call(**bad) == ALIGNMENT, bad
    query = mp8.softmax_xent_fwd_workspace_bytes if call is fwd else mp8.softmax_xent_bwd_workspace_bytes
    for dims, ld in (((300, 1000, 64), 64), ((5, 70, 33), 35)):
        need = query(*dims, ld)
        assert need > 0
        kw = dict(zip("MNK", dims), ldx=65, ldw=ld)
        if call is bwd:
            kw |= dict(dw16=P)
        assert call(ws=None, **kw) == WORKSPACE and call(n=need - 256, **kw) == WORKSPACE
    for none in (dict(M=0), dict(N=0), dict(K=0, ldx=0, ldw=0)):
        assert call(ws=None, n=0, **none) == OK
    assert query(1 << 40, 8, 8) == 0 and query(-1, 8, 8) == 0 and query(8, 8, 8, 7) == 0


def test_backward_refuses():
    assert bwd(dx16=None) == INVALID
    assert bwd(round=2) == INVALID and bwd(flags=2) == INVALID
    for bad in (dict(dx16=ODD), dict(dx8=ODD), dict(dw16=ODD), dict(dw8=ODD)):
        assert bwd(**bad) == ALIGNMENT, bad


def test_orthogonal_momentum_refuses():
    for bad in (dict(batch=-1), dict(rows=-1), dict(cols=-1), dict(w=None), dict(v=None), dict(g=None), dict(steps=0), dict(steps=65),
                dict(round=2)):
        assert ortho(**bad) == INVALID, bad
    for bad in (dict(rows=(1 << 20) + 1), dict(cols=1 << 62), dict(batch=65536), dict(rows=1 << 20, cols=1 << 20)):
        assert ortho(**bad) == UNSUPPORTED, bad
    for bad in (dict(w=ODD), dict(v=ODD), dict(g=ODD), dict(w8=ODD), dict(ws=ODD)):
        assert ortho(**bad) == ALIGNMENT, bad
    # a skip flag among the counters that the call itself adds to
    for at in (0, 4, 8, 12):
        assert ortho(stats=P, skip=C.c_void_p(4096 + at)) == INVALID
    need = mp8.orthogonal_momentum_workspace_bytes(3, 100, 50)
    assert need > 0
    for where in (C.c_void_p(4096 - 4), C.c_void_p(4096 + 16)):
        assert ortho(3, 100, 50, stats=P, skip=where, ws=None) == WORKSPACE
    assert ortho(3, 100, 50, n=need - 1) == WORKSPACE
    for none in (dict(batch=0), dict(rows=0), dict(cols=0)):
        assert ortho(ws=None, **none) == OK
    assert mp8.orthogonal_momentum_workspace_bytes(1, 1 << 40, 1) == 0


def test_the_binding_refuses():
    h, f, u, t = (torch.zeros((4, 8), dtype=d) for d in (torch.float16, torch.float32, torch.uint8, torch.int64))
    calls = [
        lambda: mp8.softmax_xent_fwd_fp16(4, 4, 8, h, h, t[:, 0].contiguous(), f[:, 0].contiguous(), f[:, 0].contiguous()),
        lambda: mp8.softmax_xent_bwd_fp16(4, 4, 8, h, h, t[:, 0].contiguous(), f[:, 0].contiguous(), f[:, 0].contiguous(), dx16=h),
        lambda: mp8.orthogonal_momentum_fp16_sr(h, f, u, 0.1, 1.0, 0.9),
    ]
    for call in calls:
        with pytest.raises(mp8.Mp8Error, match="must be a GPU tensor"):
            call()
    with pytest.raises(TypeError):
        mp8.softmax_xent_fwd_fp16(4, 4, 8, None, None, None, None, None)
    with pytest.raises(TypeError):
        mp8.orthogonal_momentum_fp16_sr(None, None, None, 0.1, 1.0, 0.9)


@pytest.mark.gpu
def test_the_binding_refuses_sizes_and_types():
    d = "cuda"
    M, N, K = 4, 6, 8
    h, w = torch.zeros((M, K), dtype=torch.float16, device=d), torch.zeros((N, K), dtype=torch.float16, device=d)
    t, f = torch.zeros(M, dtype=torch.int64, device=d), torch.zeros(M, device=d)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=d)
    with pytest.raises(mp8.Mp8Error, match="dtype"):
        mp8.softmax_xent_fwd_fp16(M, N, K, h.float(), w, t, f, f, workspace=ws)
    with pytest.raises(mp8.Mp8Error, match="dtype"):
        mp8.softmax_xent_fwd_fp16(M, N, K, h, w, t.int(), f, f, workspace=ws)
    for bad in (dict(x=h[:3]), dict(w=w[:5]), dict(t=t[:3]), dict(loss=f[:3]), dict(lse=f[:3]), dict(ldx=9), dict(ldw=9), dict(ldw=2 ** 62)):
        a = dict(x=h, w=w, t=t, loss=f, lse=f, ldx=None, ldw=None) | bad
        with pytest.raises(mp8.Mp8Error):
            mp8.softmax_xent_fwd_fp16(M, N, K, a["x"], a["w"], a["t"], a["loss"], a["lse"], workspace=ws, ldx=a["ldx"], ldw=a["ldw"])
    for bad in (dict(dx16=w), dict(dw16=h), dict(dx8=torch.zeros(5, dtype=torch.uint8, device=d)), dict(dloss=f[:2], dx16=h), dict()):
        with pytest.raises(mp8.Mp8Error):
            mp8.softmax_xent_bwd_fp16(M, N, K, h, w, t, f, f, workspace=ws, **bad)
    with pytest.raises(mp8.Mp8Error, match="workspace"):
        mp8.softmax_xent_fwd_fp16(M, N, K, h, w, t, f, f)
    v, g = torch.zeros((M, K), device=d), torch.zeros((M, K), dtype=torch.uint8, device=d)
    for bad in (dict(v=v[:3]), dict(g=g[:3]), dict(w8=g[:3]), dict(w=h.reshape(-1))):
        a = dict(w=h, v=v, g=g, w8=None) | bad
        with pytest.raises(mp8.Mp8Error):
            mp8.orthogonal_momentum_fp16_sr(a["w"], a["v"], a["g"], 0.1, 1.0, 0.9, w8_out=a["w8"], workspace=ws)
    stats = mp8.new_stats()
    with pytest.raises(mp8.Mp8Error, match="invalid"):
        mp8.orthogonal_momentum_fp16_sr(h, v, g, 0.1, 1.0, 0.9, skip_if_nonzero=stats[1:2], stats=stats, workspace=ws)
