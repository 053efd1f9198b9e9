"""Attention among all atoms of a segment, forward and backward, against 64 bits.

Tolerances (relative, in the 2-norm), u = 2^-24.  A score is a sum of D products, a few elementary operations on values up to
the largest score s in size: its error is below (sqrt(D) + 8) u s.  A weight p carries twice that (numerator and sum) and 4 u
of the exponential and the division: e = 2 (sqrt(D) + 8) u s + 4 u.  out = sum p v: e, sqrt(n) u of the sum over n keys.  The
gradients are sums of products of p, of dp - delta (a difference of sums of the same size: twice the sums' sqrt(D) u and the e
of delta), of 1 - tanh^2 and of operands: below 4 e + 4 (sqrt(D) + sqrt(n)) u.  bf16: the weights and the factors dx are rounded
to bf16 before their sums and the result once, each 2^-8 at most.  Sums whose terms cancel (slopes, places, and dq and dk where
the terms of a row sum to nothing) are measured against the norm of what they would be without cancellation: the test forms
that norm beside the reference (`size`)."""
import math

import pytest
import torch

import allpair_reference as R
from paper_2601_16622_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(dtype, D, Hq, Hk, nq, nk, biased, seed, spread=1.0, self_attention=False):
    """Segments of nq queries and nk keys; self_attention: the same atoms."""
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    Nq, Nk = sum(nq), sum(nk)
    off = lambda c: torch.tensor([0] + list(c)).cumsum(0).to(torch.int32).cuda()  # noqa: E731
    x = dict(q=(n(Nq, Hq, D) * spread).to(DT[dtype]).cuda(), k=n(Nk, Hk, D).to(DT[dtype]).cuda(), v=n(Nk, Hk, D).to(DT[dtype]).cuda(),
             q_offsets=off(nq), k_offsets=off(nk), go=n(Nq, Hq, D).to(DT[dtype]).cuda())
    if biased:
        x["k_pos"] = (n(Nk, 3) * 4).cuda()
        x["q_pos"] = x["k_pos"].clone() if self_attention else (n(Nq, 3) * 4).cuda()
        x["slope"] = (0.3 * n(Hq)).cuda()
    return x


def call(x, cap=0.0, scale=None, fill=float("nan"), backward=True, **more):
    how = dict(cap=cap, scale=scale, **{n: x.get(n) for n in ("q_pos", "k_pos", "slope", "q_lengths", "k_lengths")}, **more)
    S = x["q_offsets"].shape[0] - 1
    full = lambda t: torch.full(t.shape, fill, dtype=t.dtype, device="cuda")  # noqa: E731
    got = dict(out=full(x["q"]))
    ws = torch.empty(B.e2f_dense_attn_workspace_bytes(x["q"], x["k"], S), dtype=torch.uint8, device="cuda")
    B.e2f_dense_attn_forward(x["q"], x["k"], x["v"], x["q_offsets"], x["k_offsets"], got["out"], ws, **how)
    if not backward:
        return got
    got |= dict(q=full(x["q"]), k=full(x["k"]), v=full(x["v"]))
    if x.get("slope") is not None:
        got |= dict(slope=full(x["slope"]), q_pos=full(x["q_pos"]), k_pos=full(x["k_pos"]))
    ws = torch.empty(B.e2f_dense_attn_backward_workspace_bytes(x["q"], x["k"], S), dtype=torch.uint8, device="cuda")
    B.e2f_dense_attn_backward(x["q"], x["k"], x["v"], x["q_offsets"], x["k_offsets"], x["go"], got["q"], got["k"], got["v"], ws,
                              grad_slope=got.get("slope"), grad_q_pos=got.get("q_pos"), grad_k_pos=got.get("k_pos"), **how)
    return got


def reference(x, cap=0.0, scale=None):
    """Results, the rows that are covered, the largest score and the sizes without cancellation."""
    D, Hq, Hk = x["q"].shape[2], x["q"].shape[1], x["k"].shape[1]
    scale = D ** -0.5 if scale is None else scale
    names = [n for n in ("q", "k", "v", "slope", "q_pos", "k_pos") if x.get(n) is not None]
    t = {n: x[n].double().cpu().requires_grad_() for n in names}
    lists = {n: (x[n].tolist() if x.get(n) is not None else None) for n in ("q_offsets", "k_offsets", "q_lengths", "k_lengths")}
    out, covered = R.dense_attn(t["q"], t["k"], t["v"], scale=scale, cap=cap, **{n: t.get(n) for n in ("slope", "q_pos", "k_pos")}, **lists)
    go = x["go"].double().cpu()
    go = torch.where(covered[:, None, None], go, 0.0)
    grads = torch.autograd.grad(out, [t[n] for n in names], go, allow_unused=True)
    want = {n: (g if g is not None else torch.zeros_like(t[n])) for n, g in zip(names, grads)} | {"out": out.detach()}
    size = {n: 0.0 for n in want}
    top = 1.0
    k_covered = torch.zeros(t["k"].shape[0], dtype=torch.bool)
    for (a, n), (b, m) in zip(R.ranges(lists["q_offsets"], lists["q_lengths"], x["q"].shape[0]), R.ranges(lists["k_offsets"], lists["k_lengths"], x["k"].shape[0])):
        k_covered[b:b + m] = True
        if n == 0 or m == 0:
            continue
        for h in range(Hq):
            q, k, v, g = (z.detach() for z in (t["q"][a:a + n, h], t["k"][b:b + m, h * Hk // Hq], t["v"][b:b + m, h * Hk // Hq], go[a:a + n, h]))
            at = [z.detach() if z is not None else None for z in (t["q_pos"][a:a + n] if "slope" in t else None, t["k_pos"][b:b + m] if "slope" in t else None, t["slope"][h] if "slope" in t else None)]
            s = R.dense_scores(q, k, scale, cap, *at)
            raw = scale * (q.abs() @ k.abs().T)
            top = max(top, float(s.abs().max()), float((raw if not cap else raw.clamp(max=cap)).max()))
            p, dp = torch.softmax(s, -1), g @ v.T
            ds = p * (dp.abs() + (p * dp.abs()).sum(-1, keepdim=True))
            size["q"] += float((scale * ds @ k.abs()).square().sum())
            size["k"] += float((scale * ds.T @ q.abs()).square().sum())
            size["v"] += float((p.T @ g.abs()).square().sum())
            size["out"] += float((p @ v.abs()).square().sum())
            if "slope" in t:
                d = torch.cdist(at[0], at[1])
                size["slope"] += float((ds * d).sum()) ** 2
                size["q_pos"] += float((at[2].abs() * ds.sum(1)).square().sum())
                size["k_pos"] += float((at[2].abs() * ds.sum(0)).square().sum())
    return want, covered, k_covered, top, {n: math.sqrt(s) for n, s in size.items()}


def check(x, cap=0.0, scale=None, got=None, backward=True):
    want, covered, k_covered, top, size = reference(x, cap, scale)
    got = call(x, cap, scale, backward=backward) if got is None else got
    D, n = x["q"].shape[2], max(x["q"].shape[0] * x["q"].shape[1] // x["k"].shape[1], x["k"].shape[0])
    e = 2 * (math.sqrt(D) + 8) * U * top + 4 * U
    bf16 = 2.0 ** -8 if x["q"].dtype == torch.bfloat16 else 0.0
    for name, g in got.items():
        rows = {"out": covered, "q": covered, "q_pos": covered, "k": k_covered, "v": k_covered, "k_pos": k_covered}.get(name)
        g, w = g.double().cpu(), want[name]
        if rows is not None:
            assert bool(torch.isnan(g[~rows]).all()), name + ": rows that no segment covers"
            g, w = g[rows], w[rows]
        far = float((g - w).norm())
        # the rounding of a result counts for its own norm, everything before it for the norm without cancellation
        before = e + math.sqrt(n) * U if name == "out" else 4 * e + 4 * (math.sqrt(D) + math.sqrt(n)) * U
        if name in ("out", "q", "k", "v"):
            limit = (before + bf16) * size[name] + bf16 * float(w.norm())
        else:
            limit = before * size[name]
        assert far <= limit, (name, far, limit)


RAGGED = ([1, 0, 33, 128, 129, 64, 5], [1, 4, 31, 130, 0, 65, 257])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,Hq,Hk,nq,nk,cap,biased", [
    (8, 1, 1, [1], [1], 0.0, False), (16, 8, 8, *RAGGED, 20.0, True), (24, 4, 1, *RAGGED, 0.0, True), (32, 2, 2, [200], [1], 5.0, True),
    (48, 6, 2, *RAGGED, 3.0, False), (64, 2, 2, [300], [300], 30.0, True), (64, 8, 2, [1, 1, 1], [700, 3, 64], 30.0, True),
    (80, 3, 3, [40, 41], [100, 99], 0.0, False), (96, 4, 2, [70], [129], 10.0, True), (104, 2, 1, [65], [66], 0.0, True),
    (128, 4, 1, [33, 90], [200, 31], 50.0, True), (128, 16, 1, [9], [500], 0.0, False),
    # few rows and keys, few rows over many keys, with many features; a group of heads larger than a tile
    (128, 2, 2, [20, 30], [40, 10], 20.0, True), (96, 2, 1, [10, 0, 25], [30, 7, 64], 0.0, True), (72, 3, 3, [33, 64], [12, 33], 6.0, False),
    (128, 8, 2, [1, 2], [700, 300], 30.0, True), (88, 4, 4, [2], [1100], 0.0, False), (32, 4, 2, [3, 1], [900, 260], 10.0, True),
    (16, 200, 1, [3, 1], [40, 150], 10.0, True),
])
def test_against_64_bits(dtype, D, Hq, Hk, nq, nk, cap, biased):
    check(make(dtype, D, Hq, Hk, nq, nk, biased, D + Hq), cap)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_same_atoms_as_queries_and_keys(dtype):
    x = make(dtype, 32, 4, 4, [90, 1, 30], [90, 1, 30], True, 5, self_attention=True)
    x["k_pos"][3] = x["k_pos"][4]       # two atoms at one place: distance 0 beside that of an atom to itself
    x["q_pos"][3] = x["q_pos"][4]
    check(x, 20.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [0.0, 8.0])
def test_scores_of_many_sizes(dtype, cap):
    """Scores far beyond the cap beside scores near 0, and a softmax that falls on one key."""
    x = make(dtype, 64, 2, 1, [100], [150], True, 6, spread=30.0)
    x["q"][::3] *= 0.01
    check(x, cap, 0.4)
    x = make(dtype, 64, 2, 1, [100], [150], True, 7)
    check(x, cap, -0.2)
    check(x, cap, 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths_and_what_lies_behind_them(dtype):
    nq, nk = [40, 7, 64, 3, 20], [50, 30, 64, 8, 9]
    x = make(dtype, 32, 4, 2, nq, nk, True, 8)
    x["q_lengths"] = torch.tensor([33, 0, 64, 99, 1], dtype=torch.int32, device="cuda")      # 99: cut to the segment
    x["k_lengths"] = torch.tensor([49, 30, 1, -5, 9], dtype=torch.int32, device="cuda")      # -5: no key
    clean = call(x, 20.0)
    check(x, 20.0, got=clean)
    # whatever lies in places that do not count changes nothing
    y = {n: (t.clone() if torch.is_tensor(t) else t) for n, t in x.items()}
    for s, (a, n) in enumerate(R.ranges(x["q_offsets"].tolist(), x["q_lengths"].tolist(), sum(nq))):
        end = x["q_offsets"].tolist()[s + 1]
        for name, bad in (("q", float("nan")), ("go", float("inf")), ("q_pos", float("nan"))):
            y[name][a + n:end] = bad
    for s, (b, m) in enumerate(R.ranges(x["k_offsets"].tolist(), x["k_lengths"].tolist(), sum(nk))):
        end = x["k_offsets"].tolist()[s + 1]
        for name, bad in (("k", float("inf")), ("v", float("nan")), ("k_pos", float("inf"))):
            y[name][b + m:end] = bad
    dirty = call(y, 20.0)
    for n in clean:
        assert torch.equal(torch.nan_to_num(clean[n].float(), nan=77.0), torch.nan_to_num(dirty[n].float(), nan=77.0)), n
    z = call(x, 20.0, fill=4.0)
    assert bool((z["out"][33:40] == 4).all()) and bool((z["v"][49] == 4).all()) and bool((z["k_pos"][49] == 4).all())
    assert float(z["out"][111:114].float().abs().max()) == 0.0      # queries without keys


def test_bad_values_stay_in_their_rows():
    """A NaN in a query reaches that query's row and no other one's result; offsets beyond the tokens are cut."""
    x = make("bf16", 64, 2, 2, [100], [90], True, 9)
    want = call(x, 20.0, backward=False)["out"]
    x["q"][17, 1, 5] = float("nan")
    got = call(x, 20.0, backward=False)["out"]
    assert bool(torch.isnan(got[17, 1]).all())
    got[17, 1] = want[17, 1]
    assert torch.equal(got, want)
    y = make("f32", 16, 1, 1, [10, 20], [15, 25], False, 10)
    y["q_offsets"][2] = 2_000_000_000
    y["k_offsets"][2] = 2_000_000_000
    check(y)


def test_infinite_scores_under_a_cap():
    x = make("f32", 16, 1, 1, [5], [40], False, 11)
    x["q"][2] = 1e38
    x["k"][7] = 1e38
    x["k"][8] = -1e38
    got = call(x, 5.0, backward=False)["out"]
    assert bool(torch.isfinite(got).all())
    k, v = x["k"].double().cpu()[:, 0], x["v"].double().cpu()[:, 0]
    s = 5 * torch.tanh((x["q"].double().cpu()[2] @ k.T) * 0.25 / 5)
    assert float((got[2].double().cpu() - torch.softmax(s, -1) @ v).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    x = make(dtype, 48, 4, 2, [30, 50], [60, 20], True, 12)
    want = call(x, 20.0)
    y = dict(x)
    y["q"] = x["q"].permute(1, 0, 2).contiguous().permute(1, 0, 2)                     # heads outside
    both = torch.zeros(80, 2, 128, dtype=DT[dtype], device="cuda")                        # keys and values side by side
    both[..., :48], both[..., 64:112] = x["k"], x["v"]
    y["k"], y["v"] = both[..., :48], both[..., 64:112]
    got = call(y, 20.0)
    assert all(torch.equal(got[n], want[n]) for n in want)
    out = torch.full((4, 90, 56), 6.0, dtype=DT[dtype], device="cuda")
    view = out.permute(1, 0, 2)[3:83, :, 8:]
    B.e2f_dense_attn_forward(x["q"], x["k"], x["v"], x["q_offsets"], x["k_offsets"], view,
                             torch.empty(B.e2f_dense_attn_workspace_bytes(x["q"], x["k"], 2), dtype=torch.uint8, device="cuda"),
                             cap=20.0, q_pos=x["q_pos"], k_pos=x["k_pos"], slope=x["slope"])
    assert torch.equal(view, want["out"])
    view.fill_(6.0)
    assert bool((out == 6).all())
    # one head of keys and values for all, by a stride of 0: as with a single key head
    z = dict(x, k=x["k"][:, :1].expand(80, 4, 48), v=x["v"][:, :1].expand(80, 4, 48))
    one = dict(x, k=x["k"][:, :1].contiguous(), v=x["v"][:, :1].contiguous())
    assert torch.equal(call(z, 20.0, backward=False)["out"], call(one, 20.0, backward=False)["out"]) or dtype == "bf16"
    check(one, 20.0)


def test_gradients_that_are_not_wanted():
    x = make("bf16", 32, 2, 2, [60], [70], True, 13)
    want = call(x, 20.0)
    S, new = 1, lambda n: torch.empty_like(x[n])  # noqa: E731
    ws = torch.empty(B.e2f_dense_attn_backward_workspace_bytes(x["q"], x["k"], S), dtype=torch.uint8, device="cuda")
    for skip in range(8):
        sums = [None if skip >> i & 1 else new(n) for i, n in enumerate(("slope", "q_pos", "k_pos"))]
        g = [new(n) for n in "qkv"]
        B.e2f_dense_attn_backward(x["q"], x["k"], x["v"], x["q_offsets"], x["k_offsets"], x["go"], *g, ws, cap=20.0, q_pos=x["q_pos"], k_pos=x["k_pos"],
                                  slope=x["slope"], grad_slope=sums[0], grad_q_pos=sums[1], grad_k_pos=sums[2])
        assert all(torch.equal(a, want[n]) for a, n in zip(g, "qkv"))
        assert all(a is None or torch.equal(a, want[n]) for a, n in zip(sums, ("slope", "q_pos", "k_pos")))


@pytest.mark.parametrize("nq", [0, 20])
def test_no_queries_or_no_keys(nq):
    x = make("f32", 16, 2, 1, [nq], [20 - nq], True, 14)
    got = call(x)
    assert all(float(t.abs().max()) == 0.0 for t in got.values() if t.numel())


def test_many_segments():
    sizes = [(i * 7) % 5 for i in range(5000)]      # empty ones among them
    x = make("f32", 16, 2, 2, sizes, sizes[::-1], False, 15)
    check(x, backward=False)


def test_stream_and_graph():
    cases = [make("bf16", 64, 4, 2, [100, 30], [90, 200], True, seed) for seed in (16, 17)]
    want = [call(x, 20.0) for x in cases]
    torch.cuda.synchronize()
    buf = {n: t.clone() for n, t in cases[0].items()}
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call(buf, 20.0)
    side.synchronize()
    assert all(torch.equal(got[n], want[0][n]) for n in got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(buf, 20.0)
    for which in (1, 0, 1, 1):
        for n, t in cases[which].items():
            buf[n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[which][n]) for n in got)
        call(cases[0], 0.0)       # eager work between the replays
