"""What a program may count on from the token table's and the clip's calls, without a GPU."""
import ctypes as C

import pytest

from paper_2605_04711_b200 import binding as B


def _workspace(vocab, dim, tokens):
    e, n = B.Embed(vocab, dim, 1, 0, 0, 64, 1.0, -1, 0, 0, 0), C.c_size_t()
    assert B._lib.baoc_embed_grad_workspace_bytes(C.byref(e), tokens, C.byref(n)) == B.OK
    return n.value


@pytest.mark.parametrize("vocab,dim", [(1, 8), (300, 256), (4096, 2048), (32000, 128), (32000, 2048), (50257, 64), (50257, 512), (50257, 768),
                                       (98304, 256), (98305, 256), (128256, 64), (131072, 4096), (600000, 1), (600000, 16384)])
def test_a_workspace_serves_every_smaller_batch(vocab, dim):
    """The size never falls as the number of tokens grows: every count up to 3000, then steps that are odd and below the
    distance at which the tables' sizes move by their alignment."""
    last = 0
    for n in list(range(3000)) + list(range(3001, 300000, 37)) + [1 << 20, (1 << 20) + 1, 1 << 27, 1 << 30]:
        size = _workspace(vocab, dim, n)
        assert size >= last, n
        last = size
