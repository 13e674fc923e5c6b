"""What the binding of the softmax cross entropy and of the orthogonalised momentum refuses before anything is launched: scratch, counters and
flags in ordinary host memory, which a GPU cannot read.  Pinned memory it can."""
import pytest
import torch

from test_gpu_operator_tiles import mp8  # noqa: F401

pytestmark = pytest.mark.gpu


def calls(mp8):
    M, N, K = 4, 6, 8
    empty = lambda d, *s: torch.zeros(s, dtype=d, device="cuda")
    h, f, u = torch.float16, torch.float32, torch.uint8
    x, w, t, loss, lse, v, g = empty(h, M, K), empty(h, N, K), empty(torch.int64, M), empty(f, M), empty(f, M), empty(f, N, K), empty(u, N, K)
    return [lambda workspace: mp8.softmax_xent_fwd_fp16(M, N, K, x, w, t, loss, lse, workspace=workspace),
            lambda workspace, **kw: mp8.softmax_xent_bwd_fp16(M, N, K, x, w, t, loss, lse, dx16=empty(h, M, K), dw16=empty(h, N, K), workspace=workspace, **kw),
            lambda workspace, **kw: mp8.orthogonal_momentum_fp16_sr(w, v, g, 0.1, 1.0, 0.9, workspace=workspace, **kw)]


def test_host_memory_is_refused(mp8):
    host, device = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    words = torch.zeros(4, dtype=torch.int32)
    forward, backward, momentum = calls(mp8)
    for call in (lambda: forward(host), lambda: backward(host), lambda: momentum(host), lambda: backward(device, dx_stats=words),
                 lambda: backward(device, dw_stats=words), lambda: momentum(device, stats=words), lambda: momentum(device, skip_if_nonzero=words[:1])):
        with pytest.raises(mp8.Mp8Error, match="host memory"):
            call()


def test_a_flag_in_pinned_memory(mp8):
    device, flag = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, pin_memory=True)
    calls(mp8)[2](device, skip_if_nonzero=flag)
    torch.cuda.synchronize()
