"""Plain 64-bit forms of the operators beside the block-sparse attention, for the tests: rotary positions, the norm in front of
them, attention with a window and first tokens.  Written for reading, on torch tensors of any device."""
import math

import torch


def half_step(t):
    """Half a step of a type, relative to the value."""
    return torch.finfo(t).eps / 2


def smallest(t):
    """Half of the type's smallest step (below the normal numbers)."""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def angles(freq, pos, axis_pairs):
    """[B or 1, 1, N, pairs] in 64 bits; pos [B or 1, N, axes]."""
    axis = torch.tensor([a for a, n in enumerate(axis_pairs) for _ in range(n)], dtype=torch.long, device=freq.device)
    return (pos.double()[..., axis] * freq)[:, None]


def turn(x, angle, layout, amplitude=1.0):
    """x [B, H, N, D] in 64 bits."""
    n = 2 * angle.shape[-1]
    y = x.clone()
    first, second = (slice(0, n, 2), slice(1, n, 2)) if layout == "pairs" else (slice(0, n // 2), slice(n // 2, n))
    a, b = x[..., first], x[..., second]
    y[..., first] = amplitude * (a * torch.cos(angle) - b * torch.sin(angle))
    y[..., second] = amplitude * (a * torch.sin(angle) + b * torch.cos(angle))
    return y


def norm(x, gain, eps):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * gain


def pair_size(x, channels, layout, amplitude=1.0):
    """|first| + |second| of the pair that a channel belongs to (times the amplitude), |x| of the unturned ones."""
    y = x.abs()
    out = y.clone()
    first, second = (slice(0, channels, 2), slice(1, channels, 2)) if layout == "pairs" else (slice(0, channels // 2), slice(channels // 2, channels))
    s = abs(amplitude) * (y[..., first] + y[..., second])
    out[..., first] = s
    out[..., second] = s
    return out


def visible(rows, keys, left, right, n_sink, n_full, q_len, kv_len, device="cpu"):
    """[rows, keys] truth values of one sequence: written out row by row from the rule."""
    seen = torch.zeros((rows, keys), dtype=torch.bool, device=device)
    for i in range(min(rows, q_len)):
        p = i + kv_len - q_len
        j = torch.arange(keys, device=device)
        near = torch.ones_like(j, dtype=torch.bool)
        if left >= 0:
            near = (j >= p - left) | (j < n_sink)
        if right >= 0:
            near = near & (j <= p + right)
        seen[i] = (near | (0 <= p < n_full)) & (j < kv_len)
    return seen


def attention(q, k, v, seen, scale):
    """One head in 64 bits: q [rows, D], k, v [keys, D] -> out, lse, weights; rows that see nothing: zeros and -inf."""
    hidden = ~seen
    s = (q @ k.T * scale).masked_fill(hidden, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(hidden, 0.0, torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[:, None]))
    return p @ v, lse, p


def attention_gradients(q, k, v, out, p, dout, scale):
    """Of one head: dq, dk, dv from the formulas."""
    dp = dout @ v.T
    ds = p * (dp - (dout * out).sum(-1, keepdim=True))
    return scale * ds @ k, scale * ds.T @ q, p.T @ dout
