"""Clipping at the ends of binary32's range, against 64 bits: a factor below its normal numbers still scales to the last bit.  A value is
off by the factor's rounding and its own, 2 * 2^-24 (bf16: 2^-24 + 2^-8), or by half of the smallest number of the type (2^-150, bf16 2^-134)."""
import pytest
import torch

import allpair_reference as R
from paper_2601_16622_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e-6])
@pytest.mark.parametrize("size", [1e30, 1e37, 2e38])
def test_factors_below_the_normal_numbers(max_norm, size):
    gen = torch.Generator(device="cuda").manual_seed(3)
    grads = [(torch.rand(n, generator=gen, device="cuda") * size).to(t) for n, t in ((5003, torch.float32), (4099, torch.bfloat16), (3, torch.float32))]
    want, norm = R.clip([g.cpu() for g in grads], max_norm)
    out, got = [torch.empty_like(g) for g in grads], torch.empty(1, device="cuda")
    ws = torch.empty(B.e2f_grad_norm_clip_workspace_bytes(grads), dtype=torch.uint8, device="cuda")
    B.e2f_grad_norm_clip(grads, out, max_norm, got, ws)
    assert abs(float(got) - norm) <= U * norm or norm > 3.4e38
    for o, w in zip(out, want):
        last, least = (U, 2.0 ** -150) if o.dtype == torch.float32 else (2.0 ** -8, 2.0 ** -134)
        assert bool(((o.double().cpu() - w).abs() <= (2 * U + last) * w.abs() + least).all())
