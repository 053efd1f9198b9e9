"""Plain implementations in 64 bits of the all-pair block's operators, for the tests: loops over segments and heads,
gradients by automatic differentiation."""
import math

import torch


def qk_norm_rotate(x, weight, position, rotary_dim, layout, theta, position_scale, eps):
    """x [N][H][D] float64."""
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    y = n if weight is None else n * weight
    out = y.clone()
    for i in range(rotary_dim // 2):
        a, b = (i, i + rotary_dim // 2) if layout == "half" else (2 * i, 2 * i + 1)
        f = (position.double() * position_scale * theta ** (-2.0 * i / rotary_dim))[:, None]
        out[..., a] = y[..., a] * torch.cos(f) - y[..., b] * torch.sin(f)
        out[..., b] = y[..., b] * torch.cos(f) + y[..., a] * torch.sin(f)
    return out


def ranges(offsets, lengths, n):
    """(first, number) of the tokens of every segment."""
    got = []
    for s in range(len(offsets) - 1):
        a = min(max(offsets[s], 0), n)
        b = min(max(offsets[s + 1], a), n)
        got.append((a, b - a if lengths is None else min(max(lengths[s], 0), b - a)))
    return got


def dense_scores(q, k, scale, cap, q_pos, k_pos, slope):
    """One segment, one head: [n][m]."""
    s = scale * (q @ k.T)
    if cap > 0:
        s = cap * torch.tanh(s / cap)
    if slope is not None:
        d2 = (q_pos[:, None] - k_pos[None]).square().sum(-1)
        d = torch.where(d2 > 0, torch.sqrt(torch.where(d2 > 0, d2, 1.0)), 0.0)
        s = s - slope * d
    return s


def dense_attn(q, k, v, q_offsets, k_offsets, scale, cap=0.0, q_pos=None, k_pos=None, slope=None, q_lengths=None, k_lengths=None):
    """float64 [N][H][D] -> (out, covered rows).  Rows that no segment covers are zero and not covered."""
    group = q.shape[1] // k.shape[1]
    out, covered = torch.zeros_like(q), torch.zeros(q.shape[0], dtype=torch.bool)
    for (a, n), (b, m) in zip(ranges(q_offsets, q_lengths, q.shape[0]), ranges(k_offsets, k_lengths, k.shape[0])):
        covered[a:a + n] = True
        if n == 0 or m == 0:
            continue
        rows = []
        for h in range(q.shape[1]):
            s = dense_scores(q[a:a + n, h], k[b:b + m, h // group], scale, cap, None if slope is None else q_pos[a:a + n],
                             None if slope is None else k_pos[b:b + m], None if slope is None else slope[h])
            rows.append(torch.softmax(s, -1) @ v[b:b + m, h // group])
        out = torch.cat([out[:a], torch.stack(rows, 1), out[a + n:]])
    return out, covered


def clip(grads, max_norm):
    norm = math.sqrt(math.fsum(float((g.double() * g.double()).sum()) for g in grads))
    return [g.double() * min(1.0, max_norm / (norm + 1e-6)) for g in grads], norm
