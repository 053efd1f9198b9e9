"""The all-pair block without a GPU: the plain implementation's gradients against differences, what the entry points
refuse before anything is launched, and the workspace queries."""
import ctypes
import os

import pytest
import torch

import allpair_reference as R
from paper_2601_16622_amd import binding as B

INVALID, UNSUPPORTED, SMALL = 1, 2, 3
fake = 4096


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2601_16622_amd import build
        build.build(verbose=False)
    return B.load()


def directional(f, x, seed):
    """d/dt f(x + t u) at 0 by central differences and by the gradient: truncation h^2, rounding 2^-53 / h."""
    gen = torch.Generator().manual_seed(seed)
    u = [torch.randn(t.shape, dtype=torch.float64, generator=gen) for t in x]
    h = 1e-5
    diff = (f(*[t + h * d for t, d in zip(x, u)]) - f(*[t - h * d for t, d in zip(x, u)])) / (2 * h)
    leaves = [t.clone().requires_grad_() for t in x]
    grads = torch.autograd.grad(f(*leaves), leaves)
    return float(diff), float(sum((g * d).sum() for g, d in zip(grads, u)))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_reference_norm_gradient_against_differences(layout):
    gen = torch.Generator().manual_seed(1)
    x, w = torch.randn(3, 2, 10, dtype=torch.float64, generator=gen), torch.randn(10, dtype=torch.float64, generator=gen)
    g, pos = torch.randn(3, 2, 10, dtype=torch.float64, generator=gen), torch.tensor([0, 7, 100000])
    f = lambda x, w: (R.qk_norm_rotate(x, w, pos, 6, layout, 100.0, 0.5, 1e-6) * g).sum()  # noqa: E731
    diff, exact = directional(f, [x, w], 2)
    assert abs(diff - exact) < 1e-6 * max(1.0, abs(exact))


@pytest.mark.parametrize("cap", [0.0, 2.0])
def test_reference_attention_gradient_against_differences(cap):
    gen = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(*s, dtype=torch.float64, generator=gen)  # noqa: E731
    q, k, v, qp, kp, slope, g = n(5, 4, 8), n(7, 2, 8), n(7, 2, 8), n(5, 3), n(7, 3), n(4), n(5, 4, 8)
    f = lambda q, k, v, qp, kp, slope: (R.dense_attn(q, k, v, [0, 2, 5], [0, 4, 7], 0.7, cap, qp, kp, slope)[0] * g).sum()  # noqa: E731
    diff, exact = directional(f, [q, k, v, qp, kp, slope], 4)
    assert abs(diff - exact) < 1e-6 * max(1.0, abs(exact))


def heads(ptr=fake, token=64, head=16):
    return B.Heads(ptr, token, head)


def qk(**kw):
    a = dict(dtype=0, N=5, Hq=4, Hk=2, D=16, rotary_dim=8, layout=0, eps=1e-6, theta=1e4, position_scale=1.0, position=fake,
             weight_q=None, weight_k=None)
    a.update(kw)
    return B.QkArgs(*[a[n] for n, _ in B.QkArgs._fields_])


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), INVALID), (dict(N=-1), INVALID), (dict(Hq=-1), INVALID), (dict(D=0), INVALID), (dict(rotary_dim=7), INVALID),
    (dict(rotary_dim=18), INVALID), (dict(rotary_dim=-2), INVALID), (dict(layout=2), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(theta=0.0), INVALID), (dict(theta=float("inf")), INVALID),
    (dict(position_scale=float("inf")), INVALID), (dict(position=None), INVALID), (dict(D=12, rotary_dim=0), UNSUPPORTED),
    (dict(D=264), UNSUPPORTED), (dict(Hk=1025), UNSUPPORTED), (dict(position=fake + 2), INVALID), (dict(weight_q=fake + 1), INVALID),
])
def test_norm_refuses_bad_arguments(lib, kw, code):
    h = heads(token=1 << 14, head=264)
    assert lib.e2f_qk_norm_rotate(qk(**kw), h, h, h, h, None) == code
    assert lib.e2f_qk_norm_rotate_backward(qk(**kw), h, h, h, h, h, h, None, None, fake, 1 << 30, None) == code
    assert {"position", "weight_q"} & set(kw) or lib.e2f_qk_norm_rotate_backward_workspace_bytes(qk(**kw)) == 0


ROWS = [
    (heads(ptr=0), INVALID), (heads(token=-64), INVALID), (heads(head=-16), INVALID), (heads(ptr=fake + 4), UNSUPPORTED),
    (heads(token=66), UNSUPPORTED), (heads(head=18), UNSUPPORTED), (heads(token=1 << 62), INVALID), (heads(token=1 << 23), UNSUPPORTED),
]
RESULT_ROWS = ROWS + [(heads(token=0), INVALID), (heads(head=0), INVALID), (heads(token=16, head=16), INVALID), (heads(token=8), INVALID),
                      (heads(token=32, head=64), INVALID)]


@pytest.mark.parametrize("bad,code", ROWS)
def test_rows_that_are_read(lib, bad, code):
    good = heads()
    for at in range(2):
        rows = [good] * 4
        rows[at] = bad
        assert lib.e2f_qk_norm_rotate(qk(), *rows, None) == code
    d = dense()
    for at in range(3):
        rows = [good] * 4
        rows[at] = bad
        assert lib.e2f_dense_attn_forward(d, *rows, fake, 1 << 30, None) == code
    for at in range(4):
        rows = [good] * 7
        rows[at] = bad
        assert lib.e2f_dense_attn_backward(d, *rows, None, None, None, fake, 1 << 30, None) == code


@pytest.mark.parametrize("bad,code", RESULT_ROWS)
def test_rows_that_are_written(lib, bad, code):
    good = heads()
    for at in (2, 3):
        rows = [good] * 4
        rows[at] = bad
        assert lib.e2f_qk_norm_rotate(qk(Hk=4), *rows, None) == code
    for at in (4, 5):
        rows = [good] * 6
        rows[at] = bad
        assert lib.e2f_qk_norm_rotate_backward(qk(Hk=4), *rows, None, None, fake, 1 << 30, None) == code
    d = dense(Hk=4)
    assert lib.e2f_dense_attn_forward(d, good, good, good, bad, fake, 1 << 30, None) == code
    for at in (4, 5, 6):
        rows = [good] * 7
        rows[at] = bad
        assert lib.e2f_dense_attn_backward(d, *rows, None, None, None, fake, 1 << 30, None) == code


def dense(**kw):
    a = dict(dtype=0, Hq=4, Hk=2, D=16, Nq=5, Nk=6, S=1, scale=0.25, cap=0.0, q_offsets=fake, k_offsets=fake, q_lengths=None,
             k_lengths=None, q_pos=None, k_pos=None, slope=None)
    a.update(kw)
    return B.DenseArgs(*[a[n] for n, _ in B.DenseArgs._fields_])


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=5), INVALID), (dict(Nq=-1), INVALID), (dict(Nk=-1), INVALID), (dict(S=-1), INVALID), (dict(Hq=0), INVALID),
    (dict(Hk=0), INVALID), (dict(Hk=3), INVALID), (dict(D=0), INVALID), (dict(scale=float("nan")), INVALID), (dict(cap=-1.0), INVALID),
    (dict(cap=float("nan")), INVALID), (dict(cap=float("inf")), INVALID), (dict(cap=1e-7), UNSUPPORTED), (dict(cap=2e6), UNSUPPORTED), (dict(D=20), UNSUPPORTED), (dict(D=136), UNSUPPORTED),
    (dict(Hq=2048, Hk=1), UNSUPPORTED), (dict(q_offsets=None), INVALID), (dict(k_offsets=None), INVALID), (dict(slope=fake), INVALID),
    (dict(slope=fake, q_pos=fake), INVALID), (dict(q_pos=fake, k_pos=fake), INVALID), (dict(S=1 << 30, Hq=8, Hk=8), UNSUPPORTED),
    (dict(q_offsets=fake + 2), INVALID), (dict(k_lengths=fake + 1), INVALID), (dict(slope=fake, q_pos=fake, k_pos=fake + 2), INVALID),
])
def test_attention_refuses_bad_arguments(lib, kw, code):
    h = heads(token=1 << 14, head=136)
    assert lib.e2f_dense_attn_forward(dense(**kw), h, h, h, h, fake, 1 << 30, None) == code
    assert lib.e2f_dense_attn_backward(dense(**kw), h, h, h, h, h, h, h, None, None, None, fake, 1 << 30, None) == code


def test_attention_workspace_and_gradients_that_need_a_slope(lib):
    h, d = heads(), dense()
    need = lib.e2f_dense_attn_backward_workspace_bytes(d)
    assert need >= 5 * 4 * 16
    assert lib.e2f_dense_attn_backward_workspace_bytes(dense(slope=fake)) > need
    run = lambda d, ws, n, *sums: lib.e2f_dense_attn_backward(d, *[h] * 7, *(sums or (None,) * 3), ws, n, None)  # noqa: E731
    assert run(d, fake, need - 1) == SMALL
    assert run(d, None, need) == INVALID and run(d, fake + 16, need) == INVALID
    for at in range(3):
        sums = [None] * 3
        sums[at] = fake
        assert run(d, fake, need, *sums) == INVALID
    assert lib.e2f_dense_attn_workspace_bytes(dense(D=0)) == 0 and lib.e2f_dense_attn_backward_workspace_bytes(None) == 0


def test_empty_calls_launch_nothing(lib):
    h = B.Heads(0, 0, 0)
    assert lib.e2f_qk_norm_rotate(qk(N=0), h, h, h, h, None) == 0
    assert lib.e2f_qk_norm_rotate(qk(Hq=0, Hk=0), None, None, None, None, None) == 0
    assert lib.e2f_qk_norm_rotate_backward(qk(N=0), h, h, h, h, h, h, None, None, None, 0, None) == 0
    assert lib.e2f_dense_attn_forward(dense(Nq=0, q_offsets=None, k_offsets=None, S=0), h, heads(), heads(), h, None, 0, None) == 0
    assert lib.e2f_dense_attn_backward(dense(Nq=0, Nk=0, S=0), *[h] * 7, None, None, None, None, 0, None) == 0


def clip_call(lib, ptrs=(fake,), outs=(fake,), counts=(8,), types=(0,), max_norm=1.0, norm=fake, ws=fake, ws_bytes=1 << 20, n=None):
    m = len(ptrs)
    p = ctypes.c_void_p * m
    return lib.e2f_grad_norm_clip(m if n is None else n, p(*ptrs), p(*outs), (ctypes.c_int64 * m)(*counts), (ctypes.c_int32 * m)(*types),
                                  max_norm, norm, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), INVALID), (dict(max_norm=0.0), INVALID), (dict(max_norm=-1.0), INVALID), (dict(max_norm=float("nan")), INVALID),
    (dict(norm=None), INVALID), (dict(norm=fake + 2), INVALID), (dict(ptrs=(None,)), INVALID), (dict(outs=(None,)), INVALID),
    (dict(ptrs=(fake + 2,)), INVALID), (dict(outs=(fake + 1,), types=(1,)), INVALID), (dict(types=(3,)), INVALID),
    (dict(counts=(-1,)), INVALID), (dict(counts=(1 << 62,)), INVALID), (dict(ws=None), INVALID), (dict(ws=fake + 8), INVALID),
    (dict(ws_bytes=0), SMALL), (dict(ptrs=(fake,) * 3, outs=(fake,) * 3, counts=(8, 0, 8), types=(0, 0, 1), ws_bytes=8), SMALL),
])
def test_clipping_refuses_bad_arguments(lib, kw, code):
    assert clip_call(lib, **kw) == code


def test_clipping_workspace(lib):
    size = lambda *c: lib.e2f_grad_norm_clip_workspace_bytes(len(c), (ctypes.c_int64 * len(c))(*c))  # noqa: E731
    assert size() == 0 and size(0) == 0 and size(1) == 8 and size(-1) == 0
    assert size(1, 1, 1) == 24
    assert size(1 << 40) <= 8 * 2048 + 8
    assert size(*[1000] * 3000) == 8 * 3000


def test_binding_refuses_what_the_c_call_cannot_see(lib):
    q, k = torch.zeros(4, 2, 16), torch.zeros(4, 2, 16)
    off, out = torch.tensor([0, 4], dtype=torch.int32), torch.zeros(4, 2, 16)
    for bad in (dict(k=k.to(torch.bfloat16)), dict(k=torch.zeros(4, 2, 8)), dict(v=torch.zeros(3, 2, 16)), dict(out=out.half()),
                dict(q=torch.zeros(4, 2, 32)[..., ::2]), dict(q_offsets=off.long()), dict(k_offsets=torch.tensor([0, 2, 4], dtype=torch.int32)),
                dict(slope=torch.zeros(3)), dict(q_pos=torch.zeros(4, 2)), dict(q_lengths=torch.zeros(2, dtype=torch.int32)),
                dict(ws=torch.zeros(4)), dict()):   # at last: not on a GPU
        a = dict(q=q, k=k, v=k, q_offsets=off, k_offsets=off, out=out, ws=None) | bad
        with pytest.raises(B.E2fError) as e:
            B.e2f_dense_attn_forward(**a)
        assert e.value.code == INVALID
    for bad in (dict(k=torch.zeros(3, 2, 16)), dict(q_out=None), dict(position=torch.zeros(4)), dict(weight_q=torch.zeros(8)),
                dict(q=q.double(), q_out=q.double()), dict()):
        a = dict(q=q, k=k, q_out=out, k_out=out) | bad
        with pytest.raises(B.E2fError):
            B.e2f_qk_norm_rotate(**a)
    with pytest.raises(B.E2fError):
        B.e2f_grad_norm_clip([q], [k, k], 1.0, torch.zeros(1), None)
    with pytest.raises(B.E2fError):
        B.e2f_grad_norm_clip([q.transpose(0, 1)], [k.transpose(0, 1)], 1.0, torch.zeros(1), None)
