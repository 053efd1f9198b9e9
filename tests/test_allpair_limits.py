"""The all-pair block without a GPU: sizes at the end of what the kernels' numbers hold are refused before anything is launched."""
import os

import pytest

from paper_2601_16622_amd import binding as B
from test_allpair_host import UNSUPPORTED, dense, fake, heads

MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2601_16622_amd import build
        build.build(verbose=False)
    return B.load()


@pytest.mark.parametrize("kw", [dict(Nk=MOST), dict(Nk=MOST - 1023), dict(Nq=MOST), dict(Nq=MOST // 2, Hq=4, Hk=1)])
def test_rows_and_keys_that_a_walk_by_tiles_would_carry_past_31_bits(lib, kw):
    """A key or row counter that is a tile beyond 2^31 - 1024 would wrap and the walk not end."""
    h, d = heads(token=0), dense(**dict(dict(Hq=1, Hk=1), **kw))
    assert lib.e2f_dense_attn_workspace_bytes(d) == 0 and lib.e2f_dense_attn_backward_workspace_bytes(d) == 0
    assert lib.e2f_dense_attn_forward(d, h, h, h, heads(), fake, 1 << 62, None) == UNSUPPORTED
    assert lib.e2f_dense_attn_backward(d, h, h, h, h, heads(), heads(), heads(), None, None, None, fake, 1 << 62, None) == UNSUPPORTED
