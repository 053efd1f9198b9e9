"""The all-pair block beside the cutoff attention, as cases that can be timed and compared.

Three operators: the norms of queries and keys with the rotation by the position along a chain (kind "qk"), attention
among all atoms of a system with capped scores and a bias that falls with the distance (kind "dense"; with a few queries
of their own over each system it is the readout of a model), and the global norm and clipping of a training step's
gradients (kind "clip").

  own                  False: the plain forms; True: the library's calls
  listed()             the named cases
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  what an application holds before the call
  run(state)           one pass, its outputs in full
  work(case)           bytes and operations that the pass cannot do without
  exact(case, seed)    the outputs by definition, in 64 bits
"""
import math
import random

import torch

own = False

DENSITY = 0.1        # atoms per cubic Angstrom, as the systems of workloads.py
THETA = 10000.0
EPS = 1e-6
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the batch of small organic molecules in single precision, heads of 16 channels: the smallest calls, bound by launches
        dict(name="qk_molecules", kind="qk", dtype="f32", systems=64, lo=10, hi=60, hq=8, hk=8, D=16, rot=16, layout="half", scale=1.0, start=0, train=False),
        dict(name="dense_molecules", kind="dense", dtype="f32", systems=64, lo=10, hi=60, queries=0, hq=8, hk=8, D=16, cap=20.0, bias=True, train=False),
        # a batch of larger molecules, a training step: forward pass and every gradient
        dict(name="dense_large_train", kind="dense", dtype="bf16", systems=16, lo=150, hi=350, queries=0, hq=8, hk=8, D=64, cap=30.0, bias=True, train=True),
        # the same in single precision without a cap; the feature count of a head's invariants at degree 2
        dict(name="dense_f32_train", kind="dense", dtype="f32", systems=4, lo=700, hi=1300, queries=0, hq=8, hk=8, D=48, cap=0.0, bias=True, train=True),
        # one box of 10 000 atoms: the norms in a training step, part of the head rotated, positions far along a chain ...
        dict(name="qk_box10k_train", kind="qk", dtype="bf16", systems=1, lo=10000, hi=10000, hq=8, hk=8, D=64, rot=32, layout="half", scale=1.0, start=1000000, train=True),
        # ... the attention of a property prediction, the largest number of pairs ...
        dict(name="dense_box10k", kind="dense", dtype="bf16", systems=1, lo=10000, hi=10000, queries=0, hq=8, hk=8, D=64, cap=30.0, bias=True, train=False),
        # ... and a training step on a crop of such a box with four query heads to a key head
        dict(name="dense_box5k_train", kind="dense", dtype="bf16", systems=1, lo=5003, hi=5003, queries=0, hq=8, hk=2, D=128, cap=50.0, bias=True, train=True),
        # the largest system of the scaling runs: norms with the positions compressed for long chains, and a readout token over it
        dict(name="qk_box100k", kind="qk", dtype="bf16", systems=1, lo=100000, hi=100000, hq=16, hk=4, D=128, rot=128, layout="interleaved", scale=0.25, start=0, train=False),
        dict(name="readout_100k", kind="dense", dtype="bf16", systems=1, lo=100000, hi=100000, queries=1, hq=8, hk=2, D=64, cap=30.0, bias=True, train=False),
        # one probe atom in each of a batch of frozen surroundings
        dict(name="probes", kind="dense", dtype="f32", systems=64, lo=150, hi=350, queries=1, hq=8, hk=8, D=32, cap=20.0, bias=True, train=False),
        # the weights' gradients of four layers of the base model, as e2f_attn_backward leaves them
        dict(name="clip_layers", kind="clip", dtype="f32", layout="layers", tensors=12, elements=4 * (5 * 5 * 128 * 128 + 8 * 8 + 5 * 5), max_norm=1.0),
        # a large model's gradients in both types, pieces of two buffers with odd sizes
        dict(name="clip_large", kind="clip", dtype="mixed", layout="odd", tensors=60, elements=200_000_000, max_norm=10.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["qk", "dense", "dense", "readout", "clip"])
    if kind == "clip":
        tensors = rng.randint(2, 60)
        return dict(kind=kind, dtype=rng.choice(["f32", "bf16", "mixed"]), layout="odd", tensors=tensors, elements=_log_int(rng, 2000 * tensors, 150_000_000),
                    max_norm=rng.choice([0.5, 1.0, 10.0, 1e6]))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 1, 2, 4])
    D = rng.choice([16, 32, 48, 64, 64, 80, 128])
    train = rng.random() < 0.5
    if kind == "qk":
        systems = rng.choice([1, 1, 16, 64])
        lo = _log_int(rng, 10, 50000 // systems)
        return dict(kind=kind, dtype=dtype, systems=systems, lo=lo, hi=lo + rng.randint(0, lo), hq=hq, hk=hk, D=D, rot=rng.choice([D, D, D // 2]), layout=rng.choice(["half", "interleaved"]),
                    scale=rng.choice([1.0, 1.0, 0.125]), start=rng.choice([0, 0, 5_000_000]), train=train)
    cap = rng.choice([0.0, 20.0, 30.0, 50.0])
    bias = rng.random() < 0.75
    if kind == "readout":
        systems = rng.choice([1, 1, 4, 16, 64])
        lo = _log_int(rng, 30, 100000 // systems)
        return dict(kind="dense", dtype=dtype, systems=systems, lo=lo, hi=lo + rng.randint(0, lo // 3), queries=rng.choice([1, 1, 3, 17]), hq=hq, hk=hk, D=D, cap=cap, bias=bias, train=False)
    systems = rng.choice([1, 1, 4, 16, 64])
    most = (4000 if train else 8000) / math.sqrt(systems * hq / 8)
    lo = _log_int(rng, 5, max(6, int(0.7 * most)))
    return dict(kind=kind, dtype=dtype, systems=systems, lo=lo, hi=lo + rng.randint(0, lo // 3), queries=0, hq=hq, hk=hk, D=D, cap=cap, bias=bias, train=train)


def _sizes(case):
    """Atoms of every system of the case: a fact of the case, the same for every seed."""
    r = random.Random(case["systems"] * 1000003 + case["lo"] * 1009 + case["hi"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["systems"])]


def _pieces(case):
    """Elements and type of every gradient tensor of the case."""
    n, total = case["tensors"], case["elements"]
    if case["layout"] == "layers":
        return [(size, "f32") for _ in range(n // 3) for size in (5 * 5 * 128 * 128, 8 * 8, 5 * 5)]
    r = random.Random(n * 7919 + total)
    share = [math.exp(r.uniform(-3.0, 3.0)) for _ in range(n)]
    sizes = [max(1, int(s / sum(share) * total)) | 1 for s in share]
    return [(s, case["dtype"] if case["dtype"] != "mixed" else r.choice(["bf16", "bf16", "f32"])) for s in sizes]


def _offsets(sizes, dev):
    return torch.tensor([0] + sizes, dtype=torch.int32, device=dev).cumsum(0).to(torch.int32)


def _chain(case, sizes, dev):
    """Position of every atom along the chain of its system."""
    return case["start"] + torch.cat([torch.arange(n, device=dev, dtype=torch.int32) for n in sizes])


def _places(sizes, gen, dev):
    """Coordinates: uniform in a box of the common density for every system."""
    edge = torch.tensor([(n / DENSITY) ** (1.0 / 3.0) for n in sizes], device=dev).repeat_interleave(torch.tensor(sizes, device=dev))
    return torch.rand((sum(sizes), 3), device=dev, generator=gen) * edge[:, None]


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    if case["kind"] == "clip":
        pieces = _pieces(case)
        state, grads, outs = {"case": case, "norm": torch.empty(1, device=dev)}, [], []
        flat, done = {}, {}
        for t in ("f32", "bf16"):
            n = sum(s for s, p in pieces if p == t)
            flat[t] = (torch.randn(n, device=dev, generator=gen) * 1e-2).to(DTYPE[t])
            done[t] = (0, torch.empty_like(flat[t]))
        for size, t in pieces:
            at, out = done[t]
            g = flat[t][at:at + size]
            g.mul_(float(torch.rand(1, generator=gen, device=dev)) * 2)      # layers differ in the size of their gradients
            grads.append(g)
            outs.append(out[at:at + size])
            done[t] = (at + size, out)
        return state | {"grads": grads, "outs": outs}
    sizes = _sizes(case)
    dt, N = DTYPE[case["dtype"]], sum(sizes)
    heads = lambda n, h, s: (torch.randn((n, h, case["D"]), device=dev, generator=gen) * s).to(dt)  # noqa: E731
    if case["kind"] == "qk":
        # one projection's output holds queries and keys side by side; its scale is not that of normalised features
        both = heads(N, case["hq"] + case["hk"], 3.0)
        state = {"case": case, "q": both[:, :case["hq"]], "k": both[:, case["hq"]:], "position": _chain(case, sizes, dev)}
        for name in ("weight_q", "weight_k"):
            state[name] = 1.0 + 0.2 * torch.randn(case["D"], device=dev, generator=gen)
        if case["train"]:
            state |= {"grad_q_out": heads(N, case["hq"], 1e-2), "grad_k_out": heads(N, case["hk"], 1e-2)}
        return state
    many = [case["queries"]] * len(sizes) if case["queries"] else sizes
    Nq = sum(many)
    # normalised queries and keys with weights around 1.5: logits of a standard deviation of about 2
    state = {"case": case, "q": heads(Nq, case["hq"], 1.5), "k": heads(N, case["hk"], 1.5), "v": heads(N, case["hk"], 1.0),
             "k_offsets": _offsets(sizes, dev), "q_offsets": _offsets(many, dev), "q_pos": None, "k_pos": None, "slope": None,
             "sizes": sizes, "many": many}
    if case["bias"]:
        state["k_pos"] = _places(sizes, gen, dev)
        if case["queries"]:   # somewhere inside the system
            edge = torch.tensor([(n / DENSITY) ** (1.0 / 3.0) for n in sizes], device=dev).repeat_interleave(case["queries"])
            state["q_pos"] = torch.rand((Nq, 3), device=dev, generator=gen) * edge[:, None]
        else:
            state["q_pos"] = state["k_pos"]
        # from strong to hardly any fall with the distance over the heads, as learned from such a start
        h = torch.arange(1, case["hq"] + 1, device=dev, dtype=torch.float32)
        state["slope"] = torch.exp2(-8.0 * h / case["hq"]) * (0.8 + 0.4 * torch.rand(case["hq"], device=dev, generator=gen))
    if case["train"]:
        state["grad_out"] = heads(Nq, case["hq"], 1e-2)
    return state


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2601_16622_amd import binding as B
        return {"qk": _own_qk, "dense": _own_dense, "clip": _own_clip}[kind](B, state)
    return {"qk": _plain_qk, "dense": _plain_dense, "clip": _plain_clip}[kind](state)


# ---- the library's calls ------------------------------------------------------------------------------------------

def _own_qk(B, s):
    c, q, k = s["case"], s["q"], s["k"]
    how = dict(position=s["position"], weight_q=s["weight_q"], weight_k=s["weight_k"], rotary_dim=c["rot"], layout=c["layout"], theta=THETA, position_scale=c["scale"], eps=EPS)
    q_out, k_out = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=k.dtype, device=k.device)
    B.e2f_qk_norm_rotate(q, k, q_out, k_out, **how)
    if not c["train"]:
        return {"q": q_out, "k": k_out}
    both = torch.empty((q.shape[0], c["hq"] + c["hk"], c["D"]), dtype=q.dtype, device=q.device)
    weights = torch.empty((2, c["D"]), dtype=torch.float32, device=q.device)
    ws = torch.empty(B.e2f_qk_norm_rotate_backward_workspace_bytes(q, k), dtype=torch.uint8, device=q.device)
    B.e2f_qk_norm_rotate_backward(q, k, s["grad_q_out"], s["grad_k_out"], both[:, :c["hq"]], both[:, c["hq"]:], weights[0], weights[1], ws, **how)
    return {"q": q_out, "k": k_out, "grad": both, "grad_weights": weights}


def _own_dense(B, s):
    c, q, k, v = s["case"], s["q"], s["k"], s["v"]
    how = dict(cap=c["cap"], q_pos=s["q_pos"], k_pos=s["k_pos"], slope=s["slope"])
    out = torch.empty_like(q)
    ws = torch.empty(B.e2f_dense_attn_workspace_bytes(q, k, c["systems"]), dtype=torch.uint8, device=q.device)
    B.e2f_dense_attn_forward(q, k, v, s["q_offsets"], s["k_offsets"], out, ws, **how)
    if not c["train"]:
        return {"out": out}
    got = {"out": out, "grad_q": torch.empty_like(q), "grad_k": torch.empty_like(k), "grad_v": torch.empty_like(v)}
    if c["bias"]:
        got |= {"grad_slope": torch.empty_like(s["slope"]), "grad_q_pos": torch.empty_like(s["q_pos"]), "grad_k_pos": torch.empty_like(s["k_pos"])}
    ws = torch.empty(B.e2f_dense_attn_backward_workspace_bytes(q, k, c["systems"]), dtype=torch.uint8, device=q.device)
    B.e2f_dense_attn_backward(q, k, v, s["q_offsets"], s["k_offsets"], s["grad_out"], got["grad_q"], got["grad_k"], got["grad_v"], ws,
                              grad_slope=got.get("grad_slope"), grad_q_pos=got.get("grad_q_pos"), grad_k_pos=got.get("grad_k_pos"), **how)
    return got


def _own_clip(B, s):
    ws = torch.empty(B.e2f_grad_norm_clip_workspace_bytes(s["grads"]), dtype=torch.uint8, device=s["norm"].device)
    B.e2f_grad_norm_clip(s["grads"], s["outs"], s["case"]["max_norm"], s["norm"], ws)
    return {"grads": s["outs"], "norm": s["norm"]}


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _turn(x, cos, sin, rot, layout):
    """The first `rot` features turned by the angles; with -sin the transposed turn."""
    y, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _plain_qk(s):
    c, dt = s["case"], s["q"].dtype
    rate = c["scale"] * THETA ** (-2.0 * torch.arange(c["rot"] // 2, device=s["q"].device, dtype=torch.float64) / c["rot"])
    angle = s["position"].double()[:, None, None] * rate
    cos, sin = angle.cos().float(), angle.sin().float()

    def forward(x, w):
        x = x.float()
        return _turn(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w, cos, sin, c["rot"], c["layout"]).to(dt)

    def backward(x, w, g):
        x, g = x.float(), _turn(g.float(), cos, -sin, c["rot"], c["layout"])
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        n, u = x * r, g * w
        return (r * (u - n * (n * u).mean(-1, keepdim=True))).to(dt), (g * n).double().sum((0, 1)).float()

    got = {"q": forward(s["q"], s["weight_q"]), "k": forward(s["k"], s["weight_k"])}
    if c["train"]:
        gq, wq = backward(s["q"], s["weight_q"], s["grad_q_out"])
        gk, wk = backward(s["k"], s["weight_k"], s["grad_k_out"])
        got |= {"grad": torch.cat([gq, gk], 1), "grad_weights": torch.stack([wq, wk])}
    return got


def _padded(x, index, inside):
    """[tokens][...] as [systems][longest][...], zero behind each system's end."""
    return torch.where(inside.view(inside.shape + (1,) * (x.dim() - 1)), x[index].float(), 0.0)


def _grid(offsets, longest, n):
    at = torch.arange(longest, device=offsets.device)[None, :]
    inside = at < (offsets[1:] - offsets[:-1])[:, None]
    return torch.clamp(offsets[:-1, None] + at, max=max(n - 1, 0)).long(), inside


def _plain_dense(s):
    c, dt = s["case"], s["q"].dtype
    group, scale = c["hq"] // c["hk"], 1.0 / math.sqrt(c["D"])
    iq, mq = _grid(s["q_offsets"], max(s["many"]), s["q"].shape[0])
    ik, mk = _grid(s["k_offsets"], max(s["sizes"]), s["k"].shape[0])
    q = _padded(s["q"], iq, mq).transpose(1, 2).contiguous()                                  # [S][Hq][Lq][D]
    k = _padded(s["k"], ik, mk).transpose(1, 2).repeat_interleave(group, 1).contiguous()
    v = _padded(s["v"], ik, mk).transpose(1, 2).repeat_interleave(group, 1).contiguous()
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) * scale
    if c["cap"]:
        t = torch.tanh(x / c["cap"])
        x = c["cap"] * t
    if c["bias"]:
        gap = _padded(s["q_pos"], iq, mq)[:, :, None] - _padded(s["k_pos"], ik, mk)[:, None]  # [S][Lq][Lk][3]
        far = gap.square().sum(-1).sqrt()
        x = x - s["slope"][None, :, None, None] * far[:, None]
    x = torch.where(mk[:, None, None], x, -torch.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    got = {"out": torch.matmul(p, v).transpose(1, 2)[mq].to(dt)}
    if not c["train"]:
        return got
    go = _padded(s["grad_out"], iq, mq).transpose(1, 2).contiguous()
    shared = lambda g: g.unflatten(1, (c["hk"], group)).sum(2)  # noqa: E731
    got["grad_v"] = shared(torch.matmul(p.transpose(2, 3).contiguous(), go)).transpose(1, 2)[mk].to(dt)
    dp = torch.matmul(go, v.transpose(2, 3).contiguous())
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    if c["bias"]:
        got["grad_slope"] = -(ds * far[:, None]).double().sum((0, 2, 3)).float()
        pull = -(ds * s["slope"][None, :, None, None]).sum(1) / torch.where(far > 0, far, 1.0)
        got["grad_q_pos"] = (pull[..., None] * gap).sum(2)[mq]
        got["grad_k_pos"] = -(pull[..., None] * gap).sum(1)[mk]
    if c["cap"]:
        ds = ds * (1.0 - t * t)
    ds = ds * scale
    got["grad_q"] = torch.matmul(ds, k).transpose(1, 2)[mq].to(dt)
    got["grad_k"] = shared(torch.matmul(ds.transpose(2, 3).contiguous(), q)).transpose(1, 2)[mk].to(dt)
    return got


def _plain_clip(s):
    norm = torch.stack([g.float().square().double().sum() for g in s["grads"]]).sum().sqrt()
    factor = torch.clamp(s["case"]["max_norm"] / (norm + 1e-6), max=1.0).float()
    return {"grads": [(g.float() * factor).to(g.dtype) for g in s["grads"]], "norm": norm.float().reshape(1)}


# ---- bytes and operations -------------------------------------------------------------------------------------------

def work(case):
    if case["kind"] == "clip":
        size = sum(n * (2 if t == "bf16" else 4) for n, t in _pieces(case))
        return {"bytes": 3 * size, "flops": 3 * case["elements"]}
    sizes, b = _sizes(case), 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "qk":
        n = sum(sizes) * (case["hq"] + case["hk"]) * case["D"]
        # forward: x in, y out; backward: x and dL/dy in, dL/dx out
        return {"bytes": n * b * (5 if case["train"] else 2) + 4 * sum(sizes), "flops": n * (24 if case["train"] else 8)}
    many = [case["queries"]] * len(sizes) if case["queries"] else sizes
    pairs = sum(m * n for m, n in zip(many, sizes)) * case["hq"]
    rows, keys = sum(many) * case["hq"] * case["D"] * b, sum(sizes) * case["hk"] * case["D"] * b
    places = (sum(many) + sum(sizes)) * 12 if case["bias"] else 0
    if not case["train"]:
        return {"bytes": 2 * rows + 2 * keys + places, "flops": 4 * pairs * case["D"]}
    # backward: q, k, v and dL/dout in, three gradients out; the scores again, dP, and the three products of the gradients
    return {"bytes": 4 * rows + 6 * keys + 3 * places, "flops": 14 * pairs * case["D"]}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"qk": _exact_qk, "dense": _exact_dense, "clip": _exact_clip}[case["kind"]](case, s)


def _exact_qk(c, s):
    R = c["rot"]
    pairs = [(i, i + R // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1) for i in range(R // 2)]
    first, second = (torch.tensor([p[e] for p in pairs], device=s["q"].device) for e in (0, 1))
    turn = torch.polar(torch.ones(R // 2, dtype=torch.float64, device=s["q"].device).expand(s["q"].shape[0], 1, -1),
                       (s["position"].double() * c["scale"])[:, None, None] / THETA ** (torch.arange(0, R, 2, device=s["q"].device).double() / R))

    def f(x, w):
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["D"] + EPS) * w
        z = torch.complex(y[..., first], y[..., second]) * turn
        out = y.clone()
        out[..., first], out[..., second] = z.real, z.imag
        return out

    x = {n: s[n].double().requires_grad_(c["train"]) for n in ("q", "k", "weight_q", "weight_k")}
    got = {"q": f(x["q"], x["weight_q"]), "k": f(x["k"], x["weight_k"])}
    if c["train"]:
        g = torch.autograd.grad([got["q"], got["k"]], list(x.values()), [s["grad_q_out"].double(), s["grad_k_out"].double()])
        got |= {"grad": torch.cat(g[:2], 1), "grad_weights": torch.stack(g[2:])}
    return {n: t.detach() for n, t in got.items()}


def _exact_dense(c, s):
    names = ["q", "k", "v"] + (["slope", "q_pos", "k_pos"] if c["bias"] else [])
    full = {n: s[n].double() for n in names}
    out = torch.zeros_like(full["q"])
    grads = {n: torch.zeros_like(t) for n, t in full.items()}
    qo, ko = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    for a in range(c["systems"]):
        rq, rk = slice(qo[a], qo[a + 1]), slice(ko[a], ko[a + 1])
        for h in range(c["hq"]):
            hk = h // (c["hq"] // c["hk"])
            at = {"q": (rq, h), "k": (rk, hk), "v": (rk, hk), "slope": (h,), "q_pos": (rq,), "k_pos": (rk,)}
            x = {n: full[n][at[n]].clone().requires_grad_(c["train"]) for n in names}
            score = x["q"] @ x["k"].T / c["D"] ** 0.5
            if c["cap"]:
                score = torch.tanh(score / c["cap"]) * c["cap"]
            if c["bias"]:
                d2 = (x["q_pos"][:, None] - x["k_pos"][None]).pow(2).sum(-1)
                apart = d2 > 0
                score = score - x["slope"] * torch.where(apart, torch.where(apart, d2, 1.0).sqrt(), 0.0)
            y = torch.softmax(score, 1) @ x["v"]
            out[rq, h] = y.detach()
            if c["train"]:
                for n, g in zip(names, torch.autograd.grad(y, list(x.values()), s["grad_out"][rq, h].double())):
                    grads[n][at[n]] += g
    return {"out": out} | ({"grad_" + n: g for n, g in grads.items()} if c["train"] else {})


def _exact_clip(c, s):
    norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"]))
    factor = min(1.0, c["max_norm"] / (norm + 1e-6))
    return {"grads": [g.double() * factor for g in s["grads"]], "norm": torch.tensor([norm], dtype=torch.float64)}
