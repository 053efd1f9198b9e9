"""Global gradient norm and clipping, against 64 bits.  The sum of squares is binary64: the norm is off by its rounding to
fp32, 2^-24, and a scaled value by the factor's rounding and its own, 2 * 2^-24 (bf16: 2^-24 + 2^-8)."""
import math

import pytest
import torch

import allpair_reference as R
from paper_2601_16622_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def clip(grads, max_norm, out=None):
    out = [torch.full_like(g, 3.0) for g in grads] if out is None else out
    norm = torch.full((1,), -1.0, device="cuda")
    ws = torch.empty(B.e2f_grad_norm_clip_workspace_bytes(grads), dtype=torch.uint8, device="cuda")
    B.e2f_grad_norm_clip(grads, out, max_norm, norm, ws)
    return out, float(norm)


def check(grads, max_norm):
    want, norm = R.clip([g.cpu() for g in grads], max_norm)
    out, got = clip(grads, max_norm)
    assert abs(got - norm) <= U * norm
    for g, o, w in zip(grads, out, want):
        if norm + 1e-6 <= max_norm:
            assert torch.equal(g, o)
        else:
            last = U if g.dtype == torch.float32 else 2.0 ** -8
            assert bool(((o.double().cpu() - w).abs() <= (2 * U + last) * w.abs()).all())
    same = [g.clone() for g in grads]
    assert clip(same, max_norm, same)[1] == got
    assert all(torch.equal(a, b) for a, b in zip(same, out))


def make(sizes, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=gen, device="cuda") * scale).to(torch.bfloat16 if i % 3 == 1 else torch.float32) for i, n in enumerate(sizes)]


@pytest.mark.parametrize("sizes", [[1], [7, 0, 3], [4096, 4097, 4095], [100_001, 1, 33, 250_000], [1 + (i * 37) % 900 for i in range(400)],
                                   [0, 0], [20_000_003, 5]])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_sizes(sizes, max_norm):
    check(make(sizes, len(sizes)), max_norm)


def test_pieces_that_start_anywhere():
    for dtype in (torch.float32, torch.bfloat16):
        flat, out = torch.randn(50_000, device="cuda").to(dtype), torch.full((50_003,), 9.0, device="cuda", dtype=dtype)
        cuts = [0, 1, 8, 9, 4100, 12_345, 49_999]
        grads = [flat[a:b] for a, b in zip(cuts, cuts[1:])]
        into = [out[a + 3:b + 3] for a, b in zip(cuts, cuts[1:])]       # another alignment than the gradients
        want, norm = R.clip([g.cpu() for g in grads], 1.0)
        _, got = clip(grads, 1.0, into)
        assert abs(got - norm) <= U * norm
        last = U if dtype == torch.float32 else 2.0 ** -8
        for o, w in zip(into, want):
            assert bool(((o.double().cpu() - w).abs() <= (2 * U + last) * w.abs()).all())
        assert bool((out[:3] == 9).all()) and bool((out[50_002:] == 9).all())


def test_extreme_values():
    big = [torch.full((1000,), 2e38, device="cuda"), torch.full((10,), 1e-30, device="cuda")]
    out, norm = clip(big, 1.0)
    assert math.isinf(norm)          # beyond binary32, but the clipping is not lost
    assert float((out[0].double() - 1 / math.sqrt(1000)).abs().max()) < 1e-6
    small = [torch.full((4,), 1e-40, device="cuda"), torch.full((4,), 3e-30, device="cuda")]
    out, norm = clip(small, 1e-12)
    # squares far below binary32's range; the factor is 1e-12 / (6e-30 + 1e-6) = 1e-6 by the definition
    assert abs(norm - 6e-30) < 1e-35 and bool(((out[1].double() - 3e-36).abs() <= 4 * U * 3e-36).all())
    for bad in (float("nan"), float("inf"), -float("inf")):
        g = [torch.randn(5000, device="cuda"), torch.randn(3, device="cuda").bfloat16()]
        g[0][4321] = bad
        out, norm = clip(g, 0.1)
        assert not math.isfinite(norm) and torch.equal(out[1], g[1])
        assert torch.equal(out[0].view(torch.int32), g[0].view(torch.int32))
    g = make([1000, 1000], 3)
    out, norm = clip(g, float("inf"))
    assert torch.equal(out[0], g[0]) and abs(norm - R.clip([t.cpu() for t in g], 1.0)[1]) <= U * norm


def test_nothing_to_clip():
    assert clip([], 1.0)[1] == 0.0
    assert clip([torch.empty(0, device="cuda")], 1.0)[1] == 0.0


def test_stream_and_graph():
    a, b = make([300_000, 17, 4096], 5), make([300_000, 17, 4096], 6, 0.001)
    want = [clip(a, 1.0), clip(b, 1.0)]
    assert want[1][1] < 1.0 < want[0][1]
    buf = [g.clone() for g in a]
    out = [torch.empty_like(g) for g in a]
    norm = torch.zeros(1, device="cuda")
    ws = torch.empty(B.e2f_grad_norm_clip_workspace_bytes(buf), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.e2f_grad_norm_clip(buf, out, 1.0, norm, ws)
    side.synchronize()
    assert float(norm) == want[0][1]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.e2f_grad_norm_clip(buf, out, 1.0, norm, ws)
    for which in (1, 0, 1):
        for t, g in zip(buf, (a, b)[which]):
            t.copy_(g)
        graph.replay()
        torch.cuda.synchronize()
        assert float(norm) == want[which][1] and all(torch.equal(x, y) for x, y in zip(out, want[which][0]))
        clip(a, 0.5)
