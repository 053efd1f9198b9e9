"""Norms of queries and keys over more tokens than one launch has threads for (2^32 threads; a token of 256 features takes a row of 32 or 64)."""
import pytest
import torch

from paper_2601_16622_amd import binding as B

pytestmark = pytest.mark.gpu


def test_tokens_beyond_one_launch():
    N, D, some = (1 << 27) + 1001, 256, 1500          # 8 tokens to a workgroup of 256 threads: 2^24 workgroups and 126 more
    how = dict(rotary_dim=D, theta=10000.0, eps=1e-6)
    x = torch.zeros((N, 1, D), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = [slice(0, some), slice(N - some, N)]
    for r in rows:
        x[r] = torch.randn((some, 1, D), generator=gen, device="cuda").bfloat16()
    position = torch.arange(N, dtype=torch.int32, device="cuda")
    want = []
    for r in rows:
        want.append(torch.empty_like(x[r]))
        B.e2f_qk_norm_rotate(x[r], None, want[-1], None, position=position[r], **how)
    B.e2f_qk_norm_rotate(x, None, x, None, position=position, **how)
    for r, w in zip(rows, want):
        assert torch.equal(x[r], w)
