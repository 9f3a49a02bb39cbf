"""Plain 64-bit forms of the calls on a receiver's cache (append, read, attend),
for comparison with the kernels: loops over sequences, heads and groups."""

import numpy as np
import torch


def held_in_4_bits(x):
    """(values, codes, scales) of a 4-bit cache for x [..., D], from the
    definition: groups of 32, scale = max|x| / 7 to 5 significant bits (half up),
    code = clamp(rint(x / scale), -7, 7) + 8.  Computed in fp32 steps as the format
    defines them (numpy rounds each to nearest)."""
    x = np.asarray(x, np.float32)
    y = x.reshape(*x.shape[:-1], -1, 32)
    a = np.abs(y).max(axis=-1, keepdims=True)
    s = (a / np.float32(7)).astype(np.float32)
    s = ((s.view(np.uint32).astype(np.int64) + 0x40000) & 0xFFF80000).astype(np.uint32).view(np.float32)
    s = np.where(s < 2.0 ** -100, np.float32(0), s)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s > 0, np.clip(np.rint((y / s).astype(np.float32)), -7, 7), 0)
    return (c * s).reshape(x.shape).astype(np.float64), (c + 8).astype(np.uint8).reshape(x.shape), s[..., 0]


def pack_codes(codes):
    """[..., D] codes 0..15 -> [..., D/2] bytes in the cache's nibble order."""
    D = codes.shape[-1]
    out = np.zeros((*codes.shape[:-1], D), np.uint8)
    for c in range(D):
        g, j, i = c // 32, (c % 32) // 4, c % 4
        out[..., (D // 8) * j + 4 * g + i] = codes[..., c]
    return out[..., 0::2] | (out[..., 1::2] << 4)


def rotated(x, pos, inv_freq, norm=None, eps=1e-6):
    """x [T, heads, D] fp64, rotate-half pairs at pos * inv_freq."""
    x = np.asarray(x, np.float64)
    if norm is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(norm, np.float64)
    h = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)[None, None]
    a, b = x[..., :h], x[..., h:]
    return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)


def attend(q, k, v, causal, scale=None):
    """One sequence in fp64: q [n, Hq, D], k, v [m, H, D] -> (out, lse, sum p|v|,
    largest scale * sum |q||k| of each query)."""
    q, k, v = (torch.as_tensor(t).double() for t in (q, k, v))
    n, Hq, D = q.shape
    m, H = k.shape[0], k.shape[1]
    G = Hq // H
    scale = scale or D ** -0.5
    out = torch.zeros((n, Hq, D), dtype=torch.float64, device=q.device)
    absv = torch.zeros_like(out)
    lse = torch.full((n, Hq), -np.inf, dtype=torch.float64, device=q.device)
    size = torch.zeros((n, Hq), dtype=torch.float64, device=q.device)
    if m == 0 or n == 0:
        return out, lse, absv, size
    seen = torch.arange(m, device=q.device)[None, :] <= (m - n + torch.arange(n, device=q.device))[:, None]
    if not causal:
        seen = torch.ones_like(seen)
    some = seen.any(-1)
    for h in range(Hq):
        s = (q[:, h] @ k[:, h // G].T) * scale
        s = s.masked_fill(~seen, -np.inf)
        lse[:, h] = torch.logsumexp(s, -1)
        p = torch.softmax(s[some], -1)
        out[some, h] = p @ v[:, h // G]
        absv[some, h] = p @ v[:, h // G].abs()
        size[:, h] = ((q[:, h].abs() @ k[:, h // G].abs().T) * scale).max(-1).values
    return out, lse, absv, size


def bound(out, absv, size, dtype):
    """How far an output may be.  bf16: its own rounding (2^-9), every probability
    rounded to bf16 (2^-9 each, up to 2^-9 more in their sum), and scores summed in
    fp32 by truncation (2^-23 a product of at most 256).  fp32: scores and sums
    rounded in fp32, 2^-24 a step, exp2 within 2^-22."""
    if dtype == torch.bfloat16:
        return 2.0 ** -8 * out.abs() + (2.0 ** -8 + 2.0 ** -15 * size[..., None]) * absv + 1e-30
    return (2.0 ** -19 + 2.0 ** -20 * size[..., None]) * absv + 1e-30
