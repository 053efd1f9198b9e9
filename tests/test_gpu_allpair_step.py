"""The all-pair block's operators together, as an application runs them: a training step (norms and rotation, attention among
all atoms, both backward passes, the global norm and clipping) and a readout, against the same chain in 64 bits; whole in a
graph; on two streams at once; and with tokens beyond 32-bit offsets.

Tolerance of the chain in fp32.  The norms bring 48 * 2^-24 and the attention e = 2 (sqrt(D) + 8) 2^-24 s + 4 * 2^-24 at
scores up to s, its gradients below 4 e + 4 (sqrt(D) + sqrt(n)) 2^-24 of their norm without cancellation.  With s <= 16, D = 32,
n <= 100: e < 27 * 2^-20, the gradients below 0.7e-4 of that norm, which is below 8 times theirs here (random operands; a row's
weights sum up about 100 terms).  bf16: each rounding between two operators adds 2^-8, and 2^-8 for weights and factors inside."""
import math

import pytest
import torch

import allpair_reference as R
from paper_2601_16622_amd import binding as B

pytestmark = pytest.mark.gpu
CAP, THETA, EPS, ROT = 20.0, 1000.0, 1e-6, 16


def make(dtype, sizes, Hq, Hk, D, seed):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    N = sum(sizes)
    x = dict(qkv=n(N, Hq + 2 * Hk, D).to(dtype).cuda(), go=n(N, Hq, D).to(dtype).cuda(), pos=(3 * n(N, 3)).cuda(), wq=(1 + 0.2 * n(D)).cuda(),
             wk=(1 + 0.2 * n(D)).cuda(), slope=(0.2 * n(Hq).abs()).cuda(), position=torch.cat([torch.arange(s) for s in sizes]).to(torch.int32).cuda(),
             offsets=torch.tensor([0] + sizes).cumsum(0).to(torch.int32).cuda())
    return x, Hq, Hk


def step(x, Hq, Hk, max_norm=1e-2):
    """One training step's gradients: of the projections' rows (qkv), places, and of the parameters, clipped."""
    q, k, v = x["qkv"][:, :Hq], x["qkv"][:, Hq:Hq + Hk], x["qkv"][:, Hq + Hk:]
    new = torch.empty_like
    how = dict(position=x["position"], weight_q=x["wq"], weight_k=x["wk"], rotary_dim=ROT, theta=THETA, eps=EPS)
    S, dev = x["offsets"].shape[0] - 1, x["qkv"].device
    uq, uk, out = new(x["go"]), torch.empty(k.shape, dtype=k.dtype, device=dev), new(x["go"])
    B.e2f_qk_norm_rotate(q, k, uq, uk, **how)
    att = dict(cap=CAP, q_pos=x["pos"], k_pos=x["pos"], slope=x["slope"])
    ws = torch.empty(B.e2f_dense_attn_workspace_bytes(uq, uk, S), dtype=torch.uint8, device=dev)
    B.e2f_dense_attn_forward(uq, uk, v, x["offsets"], x["offsets"], out, ws, **att)
    grad, gq, gk = new(x["qkv"]), new(uq), new(uk)
    gs, gp, gr = new(x["slope"]), new(x["pos"]), new(x["pos"])
    ws = torch.empty(B.e2f_dense_attn_backward_workspace_bytes(uq, uk, S), dtype=torch.uint8, device=dev)
    B.e2f_dense_attn_backward(uq, uk, v, x["offsets"], x["offsets"], x["go"], gq, gk, grad[:, Hq + Hk:], ws, grad_slope=gs, grad_q_pos=gp, grad_k_pos=gr, **att)
    gwq, gwk = new(x["wq"]), new(x["wk"])
    ws = torch.empty(B.e2f_qk_norm_rotate_backward_workspace_bytes(q, k), dtype=torch.uint8, device=dev)
    B.e2f_qk_norm_rotate_backward(q, k, gq, gk, grad[:, :Hq], grad[:, Hq:Hq + Hk], gwq, gwk, ws, **how)
    params, norm = [gwq, gwk, gs], torch.empty(1, device=dev)
    ws = torch.empty(B.e2f_grad_norm_clip_workspace_bytes(params), dtype=torch.uint8, device=dev)
    B.e2f_grad_norm_clip(params, params, max_norm, norm, ws)
    return dict(out=out, qkv=grad, pos=gp + gr, wq=gwq, wk=gwk, slope=gs, norm=norm)


def reference(x, Hq, Hk, max_norm=1e-2):
    t = {n: x[n].double().cpu().requires_grad_() for n in ("qkv", "pos", "wq", "wk", "slope")}
    q, k, v = t["qkv"][:, :Hq], t["qkv"][:, Hq:Hq + Hk], t["qkv"][:, Hq + Hk:]
    pos, off = x["position"].cpu(), x["offsets"].tolist()
    uq, uk = (R.qk_norm_rotate(a, w, pos, ROT, "half", THETA, 1.0, EPS) for a, w in ((q, t["wq"]), (k, t["wk"])))
    out, _ = R.dense_attn(uq, uk, v, off, off, q.shape[2] ** -0.5, CAP, t["pos"], t["pos"], t["slope"])
    g = dict(zip(t, torch.autograd.grad(out, list(t.values()), x["go"].double().cpu())))
    clipped, norm = R.clip([g["wq"], g["wk"], g["slope"]], max_norm)
    return g | dict(zip(("wq", "wk", "slope"), clipped)) | dict(out=out.detach(), norm=torch.tensor([norm]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("Hq,Hk", [(4, 4), (4, 1)])
def test_a_training_step(dtype, Hq, Hk):
    x, Hq, Hk = make(dtype, [60, 1, 100, 37], Hq, Hk, 32, 3)
    got, want = step(x, Hq, Hk), reference(x, Hq, Hk)
    D, n, u = 32, 100, 2.0 ** -24
    e = 2 * (math.sqrt(D) + 8) * u * 16 + 4 * u
    chain = 8 * (4 * e + 4 * (math.sqrt(D) + math.sqrt(n)) * u) + 2 * 96 * u
    if dtype == torch.bfloat16:
        # uq, uk and the gradients of both are rounded, then weights, factors and results: five times 2^-8 in a gradient, which
        # meets a sum of up to 8 times its norm
        chain += 5 * 8 * 2.0 ** -8
    for name, w in want.items():
        g = got[name].double().cpu()
        assert float((g - w).norm()) <= chain * float(w.norm()), name
    assert abs(float(torch.cat([got[n] for n in ("wq", "wk", "slope")]).norm()) - 1e-2) < 1e-6


def test_a_step_in_a_graph():
    xs = [make(torch.bfloat16, [60, 1, 100, 37], 4, 2, 32, seed)[0] for seed in (4, 5)]
    want = [step(x, 4, 2) for x in xs]
    torch.cuda.synchronize()
    buf = {n: t.clone() for n, t in xs[0].items()}
    step(buf, 4, 2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(buf, 4, 2)
    for which in (1, 0, 1):
        for n, t in xs[which].items():
            buf[n].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[which][n]) for n in got)
        step(xs[0], 4, 2)


def test_two_streams_at_once():
    xs = [make(torch.bfloat16, [300, 20, 150], 8, 2, 64, seed)[0] for seed in (6, 7)]
    want = [step(x, 8, 2) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = step(xs[i], 8, 2)
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(g[n], w[n]) for n in g)


@pytest.mark.parametrize("nk,queries", [(5000, 1), (20000, 1), (3000, 5), (200, 1), (20000, 40)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_readout_equals_the_row_of_a_full_call(dtype, nk, queries):
    """A few queries over a system (keys split over waves and workgroups) against the same rows among many."""
    gen = torch.Generator().manual_seed(nk)
    n = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    q, k, v = n(queries, 4, 64).to(dtype).cuda(), n(nk, 2, 64).to(dtype).cuda(), n(nk, 2, 64).to(dtype).cuda()
    qp, kp, slope = n(queries, 3).cuda(), n(nk, 3).cuda(), n(4).abs().cuda()
    out = torch.empty_like(q)
    off = lambda m: torch.tensor([0, m], dtype=torch.int32, device="cuda")  # noqa: E731
    ws = torch.empty(B.e2f_dense_attn_workspace_bytes(q, k, 1), dtype=torch.uint8, device="cuda")
    B.e2f_dense_attn_forward(q, k, v, off(queries), off(nk), out, ws, cap=CAP, q_pos=qp, k_pos=kp, slope=slope)
    want, _ = R.dense_attn(q.double().cpu(), k.double().cpu(), v.double().cpu(), [0, queries], [0, nk], 0.125, CAP, qp.double().cpu(), kp.double().cpu(),
                           slope.double().cpu())
    # as in the attention's own tests: e, the sum over the keys, weights and result in bf16; the sum without cancellation is below sqrt(nk) times the result's norm
    u = 2.0 ** -24
    e = 2 * (8 + 8) * u * 16 + 4 * u + math.sqrt(nk) * u
    limit = e * math.sqrt(nk) + (2.0 ** -8 * 3 if dtype == torch.bfloat16 else 0.0)
    assert float((out.double().cpu() - want).norm()) <= limit * float(want.norm())


def test_tokens_beyond_32_bit_offsets():
    """A cache of over 2^32 bytes: the last segment's keys against the same keys in a small tensor, tokens and heads outside."""
    N, m, D = 18_000_000, 300, 64
    gen = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=gen).bfloat16().cuda()  # noqa: E731
    q, k, v = n(2, 4, D), n(m, 2, D), n(m, 2, D)
    q_off = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    small = torch.empty_like(q)
    B.e2f_dense_attn_forward(q, k, v, torch.tensor([0, 0, 2], dtype=torch.int32, device="cuda"), torch.tensor([0, 0, m], dtype=torch.int32, device="cuda"), small,
                             torch.empty(B.e2f_dense_attn_workspace_bytes(q, k, 2), dtype=torch.uint8, device="cuda"))
    want = small[1]
    for outside in (False, True):
        cache = torch.zeros((2, N, D) if outside else (N, 2, D), dtype=torch.bfloat16, device="cuda")
        big = cache.permute(1, 0, 2) if outside else cache
        big[N - m:] = k
        vals = big.clone(memory_format=torch.preserve_format)
        vals[N - m:] = v
        k_off = torch.tensor([0, N - m, N], dtype=torch.int32, device="cuda")
        lengths = torch.tensor([0, m], dtype=torch.int32, device="cuda")
        out = torch.empty_like(q)
        B.e2f_dense_attn_forward(q, big, vals, q_off, k_off, out, torch.empty(B.e2f_dense_attn_workspace_bytes(q, big, 2), dtype=torch.uint8, device="cuda"),
                                 k_lengths=lengths)
        assert float(out[0].float().abs().max()) == 0.0
        # another split of the keys, another order of the sums: two roundings of the result, two of the weights
        assert float((out[1].float() - want.float()).norm()) <= 4 * 2.0 ** -8 * float(want.float().norm())
        # norms and rotation of the last rows
        y = torch.empty_like(k)
        B.e2f_qk_norm_rotate(k, None, y, None)
        B.e2f_qk_norm_rotate(big, None, big, None)
        assert torch.equal(big[N - m:], y)
        del cache, big, vals
