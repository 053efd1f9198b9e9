"""Attention among all atoms of a segment: how far each value of a result may be from 64 bits, where the tests by norms see little.

Tolerance of a value, u = 2^-24 (fp32).  It is the sum of terms t_i, each a product with relative error d_i, rounded once at the end by
h (bf16 2^-8, fp32 u): |got - want| <= h |want| + sum |t_i| d_i.  In d:
  - a product of D features is off by (D + 8) u of the sum of its terms' sizes (raw), by 8 u more where a value is three bf16
    and the three smallest of the nine partial products are left out (each below 2^-22 of the product);
  - a score s that is off by that much of raw and, with a cap, by 2^-22 of the cap (the exponential form in bf16, up to a cap of 128) shifts a
    weight by twice that (the weight itself and its row's sum), and by 16 u for exponentials, distances and divisions;
  - weights and factors that enter a product are off by 2^-15 in bf16 (two bf16, the first cut, the second rounded: 2^-7 * 2^-8) and
    by 8 u in fp32, and sums over n terms by n u."""
import math

import pytest
import torch

import allpair_reference as R
from paper_2601_16622_amd import binding as B
from test_gpu_dense import DT, U, call, make, reference

pytestmark = pytest.mark.gpu


def limits(x, cap=0.0, scale=None):
    """Per value of out, q, k and v: the largest distance from 64 bits without the rounding of the result."""
    D, Hq, Hk = x["q"].shape[2], x["q"].shape[1], x["k"].shape[1]
    scale = D ** -0.5 if scale is None else scale
    bf16 = x["q"].dtype == torch.bfloat16
    q, k, v, go = (x[n].double().cpu() for n in ("q", "k", "v", "go"))
    at = [x[n].double().cpu() if x.get(n) is not None else None for n in ("q_pos", "k_pos", "slope")]
    got = dict(out=torch.zeros_like(q), q=torch.zeros_like(q), k=torch.zeros_like(k), v=torch.zeros_like(v))
    lists = {n: (x[n].tolist() if x.get(n) is not None else None) for n in ("q_offsets", "k_offsets", "q_lengths", "k_lengths")}
    for (a, n), (b, m) in zip(R.ranges(lists["q_offsets"], lists["q_lengths"], q.shape[0]), R.ranges(lists["k_offsets"], lists["k_lengths"], k.shape[0])):
        if n == 0 or m == 0:
            continue
        for h in range(Hq):
            g = h * Hk // Hq
            Q, K, V, G = q[a:a + n, h], k[b:b + m, g], v[b:b + m, g], go[a:a + n, h]
            s = R.dense_scores(Q, K, scale, cap, *((at[0][a:a + n], at[1][b:b + m], at[2][h]) if at[2] is not None else (None,) * 3))
            raw = abs(scale) * (Q.abs() @ K.abs().T)
            slack = (1 - torch.tanh(scale * (Q @ K.T) / cap).square()) if cap else 1.0
            near = (D + 16) * U * raw * slack + 16 * U * s.abs().amax() + (2.0 ** -22 * min(cap, 128.0) if bf16 else 4 * U * cap)
            d = 2 * near.amax() + 16 * U
            last = (2.0 ** -15 if bf16 else 8 * U) + max(n * Hq // Hk, m) * U
            p, A = torch.softmax(s, -1), G.abs() @ V.abs().T
            got["out"][a:a + n, h] = (d + last) * (p @ V.abs())
            got["v"][b:b + m, g] += (d + last) * (p.T @ G.abs())
            # ds = p (dp - delta): p and delta off by d and the sums over the keys, dp and delta by the products over the features
            size = p * (A + (p * A).sum(-1, keepdim=True))
            # the slack: 1 - tanh^2 at an argument that is off by its product's error, relative to it twice that, and 16 u of its own; and in the
            # reference a difference from 1 in 64 bits, off by 2^-52
            dx = size * (slack * (2 * d + last + (D + 16 + m) * U + (2 * (D + 16) * U * raw / cap if cap else 0.0) + 16 * U) + 2.0 ** -52)
            got["q"][a:a + n, h] = abs(scale) * (dx @ K.abs())
            got["k"][b:b + m, g] += abs(scale) * (dx.T @ Q.abs())
    return got


def check_values(x, cap=0.0, scale=None, rows=slice(None)):
    want, covered, k_covered, _, _ = reference(x, cap, scale)
    most, got = limits(x, cap, scale), call(x, cap, scale)
    h = 2.0 ** -8 if x["q"].dtype == torch.bfloat16 else U
    for name, e in most.items():
        w, g = want[name], got[name].double().cpu()
        ok = (g - w).abs() <= h * (w.abs() + e) + e
        ok = ok[k_covered if name in "kv" else covered][rows if name in ("out", "q") else slice(None)]
        far = ((g - w).abs() / (h * (w.abs() + e) + e))[k_covered if name in "kv" else covered]
        assert bool(ok.all()), (name, int((~ok).sum()), float(far.max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,Hk,nq,nk,cap", [
    (64, 2, 2, [300], [300], 20.0), (32, 4, 1, [200, 0, 3], [170, 9, 200], 0.0), (128, 4, 2, [150], [210], 30.0), (80, 2, 1, [100, 30], [131, 20], 50.0),
    (64, 2, 2, [20], [30], 20.0), (64, 4, 2, [1], [900], 20.0),
])
def test_every_value(dtype, D, Hq, Hk, nq, nk, cap):
    check_values(make(dtype, D, Hq, Hk, nq, nk, True, D + Hq + len(nq)), cap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [2.0 ** -20, 0.5, 127.0, 129.0, 1e3, 2.0 ** 14, 1e5, 2.0 ** 20])
def test_caps_over_the_whole_range(dtype, cap):
    """Scores of a usual size under every cap that is accepted: many rows, few rows, and few rows over many keys."""
    for nq, nk in (([200], [260]), ([20], [40]), ([1], [600])):
        check_values(make(dtype, 64, 2, 1, nq, nk, True, 31), cap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("level", [1.5, 4.0, 6.0, 7.5, 9.0, 12.0])
def test_scores_at_the_cap(dtype, sign, level):
    """Queries along or against all keys, every score near +-cap: 1 - tanh^2 is small there and grad_q and grad_k are products with it."""
    x = make(dtype, 32, 2, 1, [70], [90], True, 32)
    cap, base = 10.0, torch.randn(32, generator=torch.Generator().manual_seed(1)).cuda()
    x["k"] = (base + 0.05 * x["k"].float()).to(DT[dtype])
    x["q"] = (sign * level * cap * 32 ** 0.5 * base / base.square().sum() + 0.05 * x["q"].float()).to(DT[dtype])
    check_values(x, cap)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq,nk", [(80, 100), (5, 20), (1, 700), (300, 700)])
@pytest.mark.parametrize("far", [1e19, 3e38, float("inf"), -float("inf")])
def test_keys_far_away_are_as_keys_that_are_not_there(dtype, nq, nk, far):
    """With a slope of 0.3 a key beyond 1e19 has weight 0: bit for bit as behind its segment's length.  Without one its weight is that of its product."""
    x = make(dtype, 32, 2, 1, [nq], [nk], True, 33)
    x["slope"] = torch.full_like(x["slope"], 0.3)
    gone = dict(x, k_lengths=torch.tensor([nk - 3], dtype=torch.int32, device="cuda"))
    want = call(gone, 20.0, fill=0.0)
    y = dict(x, k_pos=x["k_pos"].clone())
    y["k_pos"][nk - 3:] = far
    y["k_pos"][nk - 1, 1:] = 1.0
    got = call(y, 20.0)
    for n in want:
        assert torch.equal(got[n], want[n]), n
    y["slope"] = x["slope"] * torch.tensor([0.0, 1.0], device="cuda")
    got, plain = call(y, 20.0), call(dict(x, q_pos=None, k_pos=None, slope=None), 20.0)
    assert torch.equal(got["out"][:, 0], plain["out"][:, 0]) and torch.equal(got["out"][:, 1], want["out"][:, 1])
    assert all(bool(torch.isfinite(t).all()) for n, t in got.items())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_query_far_away_reaches_no_other_row(dtype):
    """Its own scores of 1e18 have lost what tells keys apart; rows beside it have not."""
    x = make(dtype, 32, 2, 2, [80], [100], True, 34)
    want = call(x, 20.0)
    x["q_pos"][11] = torch.tensor([1e30, -float("inf"), 2.0], device="cuda")
    got = call(x, 20.0)
    for n in ("out", "q", "q_pos"):
        assert torch.equal(got[n][:11], want[n][:11]) and torch.equal(got[n][12:], want[n][12:])
    x["q_pos"][11, 0] = float("nan")
    got = call(x, 20.0, backward=False)["out"]
    assert bool(torch.isnan(got[11]).all()) and torch.equal(got[12:], want["out"][12:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 96])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_entries_that_are_not_finite_stay_in_what_they_enter(dtype, D, bad):
    x = make(dtype, D, 2, 1, [60, 70], [80, 50], True, 35)
    want = call(x, 20.0)
    segment = {n: 60 if n in ("out", "q", "q_pos") else 80 for n in want if n != "slope"}
    y = dict(x, q=x["q"].clone())
    y["q"][7, 1, 3] = bad
    got = call(y, 20.0)
    for n in ("out", "q"):
        assert torch.equal(got[n][:, 0], want[n][:, 0]) and torch.equal(got[n][:7], want[n][:7]) and torch.equal(got[n][8:], want[n][8:]), n
    assert all(torch.equal(got[n][b:], want[n][b:]) for n, b in segment.items())
    for name, at in (("k", 80 + 3), ("v", 80 + 3), ("go", 60 + 3)):
        y = dict(x, **{name: x[name].clone()})
        y[name][at, 0, 5] = bad
        got = call(y, 20.0)
        assert all(torch.equal(got[n][:b], want[n][:b]) for n, b in segment.items()), name
        if name == "go":
            assert torch.equal(got["out"], want["out"])
        if name == "v":
            assert not bool(torch.isfinite(got["out"][60:, :, 5]).any())
