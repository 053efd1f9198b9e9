"""The all-pair block without a GPU: sizes at the end of what the kernels' numbers hold are refused before anything is launched."""
import os

import pytest
import torch

from paper_2601_16622_amd import binding as B
from test_allpair_host import INVALID, UNSUPPORTED, dense, fake, heads, qk

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


@pytest.mark.parametrize("kw", [dict(S=1 << 27, Nq=1 << 27, Nk=1 << 27), dict(S=1 << 23, Nq=1 << 30, Nk=1 << 30, Hq=2, Hk=2)])
def test_more_workgroups_than_a_launch_takes(lib, kw):
    """2^32 threads along a grid's first axis; 2^27 segments of a wave each are 2^33."""
    h, d = heads(token=0), dense(**dict(dict(Hq=1, Hk=1), **kw))
    assert lib.e2f_dense_attn_workspace_bytes(d) == 0 and lib.e2f_dense_attn_backward_workspace_bytes(d) == 0
    assert lib.e2f_dense_attn_forward(d, h, h, h, heads(), fake, 1 << 62, None) == UNSUPPORTED
    assert lib.e2f_dense_attn_backward(d, h, h, h, h, heads(), heads(), heads(), None, None, None, fake, 1 << 62, None) == UNSUPPORTED


def test_sizes_that_the_header_says_pass(lib):
    n, m = (1 << 29) - 1, (1 << 22) - 1
    for kw in (dict(Nq=n, Nk=n, S=m), dict(Nq=n // 8, Nk=n // 8, Hq=8, Hk=8, S=m // 8, D=128), dict(Nq=n // 8, Nk=n, Hq=8, S=m), dict(Nq=m * 8, Nk=m * 65, S=m, dtype=1),
               dict(Nq=m * 32, Nk=n, S=m), dict(Nq=n, Nk=m * 64, S=m)):
        assert lib.e2f_dense_attn_backward_workspace_bytes(dense(**dict(dict(Hq=1, Hk=1), **kw))) > 0


@pytest.mark.parametrize("k", [torch.zeros(16), torch.zeros(4, 16), torch.zeros(())])
def test_binding_refuses_keys_of_another_rank(lib, k):
    q = torch.zeros(4, 2, 16)
    for call in (lambda: B.e2f_qk_norm_rotate(q, k, q, k), lambda: B.e2f_qk_norm_rotate_backward(q, k, q, k, q, k, None, None, None),
                 lambda: B.e2f_qk_norm_rotate_backward_workspace_bytes(q, k), lambda: B.e2f_dense_attn_workspace_bytes(q, k, 1)):
        with pytest.raises(B.E2fError) as e:
            call()
        assert e.value.code == B.E2F_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(position_scale=1e300), dict(position_scale=-1e299), dict(theta=1e-300, rotary_dim=16, position_scale=1e100), dict(theta=5e-324, rotary_dim=16, position_scale=1e50)])
def test_angles_beyond_binary64(lib, kw):
    """Infinite angles made every rotated feature a NaN."""
    h = heads()
    assert lib.e2f_qk_norm_rotate_backward_workspace_bytes(qk(**kw)) == 0
    assert lib.e2f_qk_norm_rotate_backward(qk(**kw), h, h, h, h, h, h, None, None, fake, 1 << 30, None) == INVALID
    assert lib.e2f_qk_norm_rotate(qk(**kw), h, h, h, h, None) == INVALID


@pytest.mark.parametrize("kw", [dict(theta=0.5), dict(theta=1e300), dict(position_scale=1e200, rotary_dim=0), dict(theta=1e-3, rotary_dim=2)])
def test_angles_within_binary64(lib, kw):
    assert lib.e2f_qk_norm_rotate_backward_workspace_bytes(qk(**kw)) > 0
