"""Norms of queries and keys with the rotation along the chain, forward and backward, against 64 bits.

Tolerances.  u = 2^-24 (fp32).  A forward value is x r w c + x' r w' s: r carries half the error of a D-term sum of squares
(formed in lanes of at most 8 terms and log2 exchanges: at most 16 u) and 3 roundings, the products 4 and the angle's cos and
sin one unit of the last place and the rounding of the reduced angle, 2 pi 2^-25: below 32 u of the two terms' norm, which is at most
sqrt(2) of the result's: 48 u.  A backward value adds the same sums again and the difference w g - n mean: 96 u.  bf16 adds one rounding of
the result, 2^-8.  dw sums N H products of relative error 48 u with random signs; in the worst case the sum's norm is that of one term in
sqrt(N H), so 48 u sqrt(N H) bounds what the terms bring, and pairwise sums of at most N H / 4 terms in binary32 add no more."""
import math

import pytest
import torch

import allpair_reference as R
from paper_2601_16622_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def rel(a, b):
    a, b = a.double().cpu(), b.double().cpu()
    return float((a - b).norm() / b.norm()) if float(b.norm()) else float((a - b).abs().max()) if a.numel() else 0.0


def make(dtype, N, Hq, Hk, D, seed, start=0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen).to(DT[dtype]).cuda()  # noqa: E731
    x = dict(q=n(N, Hq, D), k=n(N, Hk, D), gq=n(N, Hq, D), gk=n(N, Hk, D))
    x["position"] = (start + torch.randint(0, 5000, (N,), generator=gen)).to(torch.int32).cuda()
    x["wq"], x["wk"] = 1 + 0.3 * torch.randn(D, generator=gen).cuda(), 1 + 0.3 * torch.randn(D, generator=gen).cuda()
    return x


def run(x, weights=True, how=None, q=True, k=True):
    how = dict(how, position=x["position"], weight_q=x["wq"] if weights else None, weight_k=x["wk"] if weights else None)
    full = lambda t, on: torch.full(t.shape, float("nan"), dtype=t.dtype, device=t.device) if on else None  # noqa: E731
    a, b = x["q"] if q else None, x["k"] if k else None
    out = dict(q=full(x["q"], q), k=full(x["k"], k), dq=full(x["q"], q), dk=full(x["k"], k), dwq=torch.full_like(x["wq"], 7.0), dwk=torch.full_like(x["wk"], 7.0))
    B.e2f_qk_norm_rotate(a, b, out["q"], out["k"], **how)
    ws = torch.empty(B.e2f_qk_norm_rotate_backward_workspace_bytes(a, b), dtype=torch.uint8, device="cuda")
    B.e2f_qk_norm_rotate_backward(a, b, x["gq"] if q else None, x["gk"] if k else None, out["dq"], out["dk"], out["dwq"], out["dwk"], ws, **how)
    return out


def reference(x, weights, how, n):
    t = x[n].double().cpu().requires_grad_()
    w = x["w" + n].double().cpu().requires_grad_()
    y = R.qk_norm_rotate(t, w if weights else torch.ones_like(w) * w.detach() * 0 + 1 + (w - w.detach()), x["position"].cpu(), how["rotary_dim"], how["layout"],
                         how["theta"], how["position_scale"], how["eps"])
    dt, dw = torch.autograd.grad(y, [t, w], x["g" + n].double().cpu())
    return y.detach(), dt, dw


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,Hq,Hk,D,rot,layout", [
    (1, 1, 1, 8, 8, "half"), (1, 8, 2, 64, 64, "half"), (77, 4, 4, 64, 32, "half"), (130, 3, 1, 48, 48, "half"), (33, 2, 2, 80, 20, "half"),
    (65, 2, 2, 40, 6, "half"), (257, 8, 8, 16, 16, "interleaved"), (100, 5, 1, 128, 2, "interleaved"), (19, 2, 1, 256, 256, "interleaved"),
    (61, 1, 2, 256, 128, "half"), (300, 4, 2, 24, 0, "half"), (5001, 2, 1, 32, 32, "half"), (66, 2, 2, 200, 90, "interleaved"),
])
def test_against_64_bits(dtype, N, Hq, Hk, D, rot, layout):
    x = make(dtype, N, Hq, Hk, D, N + D)
    how = dict(rotary_dim=rot, layout=layout, theta=10000.0, position_scale=1.0, eps=1e-6)
    weights = N != 77
    got = run(x, weights, how)
    last = 2.0 ** -8 if dtype == "bf16" else 0.0
    for n, heads in (("q", Hq), ("k", Hk)):
        y, dt, dw = reference(x, weights, how, n)
        assert rel(got[n], y) <= 48 * U + last
        assert rel(got["d" + n], dt) <= 96 * U + last
        assert rel(got["dw" + n], dw) <= 48 * U * math.sqrt(N * heads)


@pytest.mark.parametrize("start,scale", [(0, 0.125), (2_000_000_000, 1.0), (-1_000_000, 1.0)])
def test_far_positions_and_scaled_ones(start, scale):
    x = make("f32", 64, 2, 1, 64, 5, start)
    how = dict(rotary_dim=64, layout="half", theta=500.0, position_scale=scale, eps=1e-5)
    got = run(x, True, how)
    # the angle itself is a product of 64 bits: 2^-53 of up to 2e9 radians, below 2^-22
    assert rel(got["q"], reference(x, True, how, "q")[0]) <= 48 * U + 2.0 ** -22


def test_one_side_alone_and_in_place():
    x = make("bf16", 90, 4, 2, 64, 9)
    how = dict(rotary_dim=24, layout="half", theta=10000.0, position_scale=1.0, eps=1e-6)   # partners read from memory
    both = run(x, True, how)
    q, k = run(x, True, how, k=False), run(x, True, how, q=False)
    assert torch.equal(q["q"], both["q"]) and torch.equal(k["k"], both["k"]) and torch.equal(k["dk"], both["dk"])
    assert float(q["dwk"].abs().max()) == 0.0 and float(k["dwq"].abs().max()) == 0.0
    assert rel(q["dwq"], both["dwq"]) <= 48 * U * math.sqrt(90 * 4)
    how = dict(how, position=x["position"], weight_q=x["wq"], weight_k=x["wk"])
    a, b, ga, gb = (x[n].clone() for n in ("q", "k", "gq", "gk"))
    ws = torch.empty(B.e2f_qk_norm_rotate_backward_workspace_bytes(a, b), dtype=torch.uint8, device="cuda")
    B.e2f_qk_norm_rotate_backward(a, b, ga, gb, ga, gb, None, None, ws, **how)
    B.e2f_qk_norm_rotate(a, b, a, b, **how)
    assert torch.equal(a, both["q"]) and torch.equal(b, both["k"]) and torch.equal(ga, both["dq"]) and torch.equal(gb, both["dk"])


def test_strides_and_neighbouring_memory():
    how = dict(rotary_dim=32, layout="interleaved", theta=10000.0, position_scale=1.0, eps=1e-6)
    x = make("f32", 50, 3, 3, 40, 11)
    want = run(x, True, how)
    base = torch.full((3, 50, 48), 5.0, device="cuda")          # heads outside, room between the rows
    y = dict(x)
    y["q"] = base.permute(1, 0, 2)[..., :40]
    y["q"].copy_(x["q"])
    got = run(y, True, how)
    assert torch.equal(got["q"], want["q"]) and torch.equal(got["dq"], want["dq"])
    out = torch.full((3, 50, 48), 5.0, device="cuda")
    B.e2f_qk_norm_rotate(x["q"], x["k"], out.permute(1, 0, 2)[..., 4:44], torch.empty_like(x["k"]), position=x["position"], weight_q=x["wq"], weight_k=x["wk"], **how)
    assert torch.equal(out.permute(1, 0, 2)[..., 4:44], want["q"])
    assert bool((out[..., :4] == 5).all()) and bool((out[..., 44:] == 5).all())
    # one head's rows for all heads (stride 0), gradients of zero rows
    one = x["q"][:, :1].expand(50, 3, 40)
    z = dict(x, q=one)
    got = run(z, True, how)
    assert torch.equal(got["q"][:, 2], want["q"][:, 0]) and torch.equal(got["q"][:, 1], want["q"][:, 0])
    zero = dict(x, q=torch.zeros_like(x["q"]))
    got = run(zero, True, how)
    assert float(got["q"].abs().max()) == 0.0 and bool(torch.isfinite(got["dq"]).all()) and float(got["dwq"].abs().max()) == 0.0


def test_no_tokens():
    x = make("f32", 0, 2, 1, 16, 1)
    got = run(x, True, dict(rotary_dim=16, layout="half", theta=100.0, position_scale=1.0, eps=1e-6))
    assert float(got["dwq"].abs().max()) == 0.0 and float(got["dwk"].abs().max()) == 0.0


def test_stream_and_graph():
    how = dict(rotary_dim=32, layout="half", theta=10000.0, position_scale=1.0, eps=1e-6)
    x, y = make("bf16", 200, 4, 2, 64, 21), make("bf16", 200, 4, 2, 64, 22)
    want = [run(x, True, how), run(y, True, how)]
    torch.cuda.synchronize()
    buf = {n: t.clone() for n, t in x.items()}
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = run(buf, True, how)
    side.synchronize()
    assert all(torch.equal(got[n], want[0][n]) for n in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(buf, True, how)
    for which in (1, 0, 1, 1):
        for n, t in (x, y)[which].items():
            buf[n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[which][n]) for n in got)
        run(x, True, how)      # eager work between the replays
