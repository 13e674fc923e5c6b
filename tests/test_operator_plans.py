"""How the softmax cross entropy and the orthogonalised momentum cut their work: what the workspace queries show of it."""
import pytest

import paper_1905_12334_amd as mp8


def up(n, to):
    return -(-n // to) * to


@pytest.mark.parametrize("M,N,K", [(1 << 20, 1 << 19, 64), (1 << 21, 1 << 18, 256), (1 << 18, 1 << 21, 8), (1 << 17, 1 << 22, 128), (1 << 22, 1 << 17, 512),
                                   (1 << 22, (1 << 17) - 300, 8), (1 << 19, 1 << 19, 64), (4096, 32000, 512), (1 << 22, 2, 8)])
def test_logits_in_one_launch(M, N, K):
    """A launch holds less than 2^32 threads: up to 2^24 - 1 workgroups of 256 of them.  The forward pass keeps eight bytes per token and tile of
    logits, beside a copy of x and four bytes per token."""
    parts, rest = divmod(mp8.softmax_xent_fwd_workspace_bytes(M, N, K) - up(2 * M * up(K, 64), 256) - up(4 * M, 256), 8 * M)
    tiles = [t for t in (64, 128, 256) if -(-N // t) == parts]
    assert tiles and rest < 256
    assert -(-M // min(tiles)) * parts <= 1 << 23


@pytest.mark.parametrize("M,N,K,share", [(8192, 131072, 2048, 32), (6007, 37003, 1000, 32), (4096, 32000, 512, 16), (1 << 17, 1 << 20, 64, 16),
                                         (512, 1000, 64, 8), (1, 32000, 512, 8)])
def test_forward_workspace_as_stated(M, N, K, share):
    """M * N / 8 bytes, and M * N / 16 or / 32 where larger tiles are taken: up to one tile of classes more, beside the copy of x and four bytes
    per token."""
    need = mp8.softmax_xent_fwd_workspace_bytes(M, N, K) - up(2 * M * up(K, 64), 256) - up(4 * M, 256)
    assert M * N // share <= need <= M * N // share + 8 * M + 256
