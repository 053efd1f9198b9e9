"""Attention among all atoms of a segment where its loops are cut into parts and many segments share a call: the forms that training steps of one
large system take, against 64 bits, with rows and keys that no length covers beside the joins.  Tolerances: tests of every value (norms for
sums over all pairs)."""
import pytest
import torch

from paper_2601_16622_amd import binding as B
from test_gpu_dense import DT, call, check, make
from test_gpu_dense_accuracy import check_values

pytestmark = pytest.mark.gpu
DTYPES = ["bf16", "f32"]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,Hq,Hk,nq,nk,cap", [
    (128, 8, 2, [700], [1300], 50.0), (80, 4, 2, [600], [600], 30.0), (48, 2, 2, [1100], [1100], 0.0), (64, 8, 8, [900], [800], 30.0),
    (96, 4, 1, [520], [1030], 20.0), (32, 2, 1, [1500], [513], 0.0), (128, 2, 2, [40], [1500], 30.0), (64, 6, 2, [1000], [30], 20.0),
    (128, 4, 4, [700, 0, 900], [1000, 600, 800], 30.0),
])
def test_loops_in_parts(dtype, D, Hq, Hk, nq, nk, cap):
    x = make(dtype, D, Hq, Hk, nq, nk, True, D + Hq)
    check(x, cap)
    check_values(x, cap)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [32, 64, 80, 128])
def test_parts_beside_rows_and_keys_that_do_not_count(dtype, D):
    """Joins leave what no segment's length covers, and parts without keys or rows bring nothing."""
    x = make(dtype, D, 4, 2, [700, 5, 0, 800], [1600, 0, 40, 1700], True, D)
    x["q_lengths"] = torch.tensor([690, 5, 0, 10], dtype=torch.int32, device="cuda")
    x["k_lengths"] = torch.tensor([300, 0, 40, 1650], dtype=torch.int32, device="cuda")
    check(x, 20.0)
    check_values(x, 20.0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_the_same_call_again_has_the_same_bits(dtype):
    x = make(dtype, 128, 8, 2, [700], [1300], True, 3)
    want = call(x, 30.0)
    for _ in range(3):
        got = call(x, 30.0, fill=1.0)
        assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("S", [63, 64, 65, 200, 5000])
def test_many_segments_both_ways(dtype, S):
    """A workgroup finds its segment among up to 63 in one round, in more rounds beyond; with lengths, and with empty segments."""
    nq, nk = [(i * 7) % 5 for i in range(S)], [(i * 3) % 6 for i in range(S)]
    nq[S // 2], nk[S // 3], nk[S // 2] = 150, 140, 70
    x = make(dtype, 16, 2, 1, nq, nk, True, S)
    check(x, 10.0)
    gen = torch.Generator().manual_seed(S)
    x["q_lengths"], x["k_lengths"] = ((torch.tensor(n) - torch.randint(0, 3, (S,), generator=gen)).to(torch.int32).cuda() for n in (nq, nk))
    check(x, 10.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("nk", [80, 700])
def test_keys_and_values_at_a_stride_of_zero(dtype, nk):
    """One head's rows for all heads, and one token's rows for all tokens: the views themselves against 64 bits, both ways."""
    x = make(dtype, 48, 4, 4, [70], [nk], True, 12)
    heads = dict(x, k=x["k"][:, :1].expand(nk, 4, 48), v=x["v"][:, :1].expand(nk, 4, 48), q=x["q"][:, 1:2].expand(70, 4, 48))
    tokens = dict(x, k=x["k"][:1].expand(nk, 4, 48), v=x["v"][3:4].expand(nk, 4, 48), go=x["go"][5:6].expand(70, 4, 48))
    for y in (heads, tokens):
        assert 0 in y["k"].stride() and 0 in y["v"].stride()
        z = {n: (t.contiguous() if n in ("q", "k", "v", "go") else t) for n, t in y.items()}
        results = dict(q=torch.empty_like(z["q"]), k=torch.empty_like(z["k"]), v=torch.empty_like(z["v"]))
        how = dict(cap=20.0, q_pos=y["q_pos"], k_pos=y["k_pos"], slope=y["slope"])
        sums = dict(grad_slope=torch.empty_like(y["slope"]), grad_q_pos=torch.empty_like(y["q_pos"]), grad_k_pos=torch.empty_like(y["k_pos"]))
        out = torch.empty_like(z["q"])
        ws = torch.empty(max(B.e2f_dense_attn_workspace_bytes(y["q"], y["k"], 1), B.e2f_dense_attn_backward_workspace_bytes(y["q"], y["k"], 1)), dtype=torch.uint8, device="cuda")
        B.e2f_dense_attn_forward(y["q"], y["k"], y["v"], y["q_offsets"], y["k_offsets"], out, ws, **how)
        B.e2f_dense_attn_backward(y["q"], y["k"], y["v"], y["q_offsets"], y["k_offsets"], y["go"], results["q"], results["k"], results["v"], ws, **sums, **how)
        got = dict(out=out, slope=sums["grad_slope"], q_pos=sums["grad_q_pos"], k_pos=sums["grad_k_pos"], **results)
        check(z, 20.0, got=got)
        want = call(z, 20.0)
        assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_workspace_for_calls_in_turn(dtype):
    """Calls of other sizes before it leave their statistics and parts in the workspace: nothing of them is read."""
    cases = [make(dtype, D, 4, 2, [n], [m], True, D) for D, n, m in ((128, 700, 900), (32, 50, 60), (64, 600, 1000))]
    want = [call(x, 20.0) for x in cases]
    S = 1
    size = max(max(B.e2f_dense_attn_workspace_bytes(x["q"], x["k"], S), B.e2f_dense_attn_backward_workspace_bytes(x["q"], x["k"], S)) for x in cases)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")        # NaN to begin with
    for x, w in list(zip(cases, want)) * 2:
        how = dict(cap=20.0, q_pos=x["q_pos"], k_pos=x["k_pos"], slope=x["slope"])
        got = {n: torch.full_like(t, 5.0) for n, t in w.items()}
        B.e2f_dense_attn_forward(x["q"], x["k"], x["v"], x["q_offsets"], x["k_offsets"], got["out"], ws, **how)
        B.e2f_dense_attn_backward(x["q"], x["k"], x["v"], x["q_offsets"], x["k_offsets"], x["go"], got["q"], got["k"], got["v"], ws,
                                  grad_slope=got["slope"], grad_q_pos=got["q_pos"], grad_k_pos=got["k_pos"], **how)
        assert all(torch.equal(got[n], w[n]) for n in w)
