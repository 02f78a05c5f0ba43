"""Rotary positions and the norm in front of them in 64 bits, from their definitions, with how far fp32 arithmetic may be off for every single value.

u = 2^-24 is half a step of fp32.  An angle: turns = position x (frequency / 2 pi) in double, three roundings; what is left of a turn is rounded to fp32, 2^-26 turns at most;
sine and cosine are within 2 steps.  All of it shifts a result by at most angle_off x the pair's magnitudes."""
import math

import torch

U = 2.0 ** -24


def turn(x, freq, axis, positions, interleaved, magnitude, back=False):
    """(rotated x, how far fp32 may be off) of x [B, H, N, d]; positions [N, axes] or [B, N, axes]."""
    x, freq = x.double().cpu(), freq.double().cpu()
    n = len(freq)
    axis = torch.zeros(n, dtype=torch.int64) if axis is None else axis.long().cpu()
    at = positions.cpu().double()[..., axis]
    at = at[None, None] if at.dim() == 2 else at[:, None]
    angle = at * freq
    angle_off = 2 * math.pi * 2.0 ** -26 + 4 * 2 * U + angle.abs() * 4 * 2.0 ** -53
    c, s = torch.cos(angle) * magnitude, torch.sin(angle) * magnitude * (-1 if back else 1)
    first = torch.arange(n) * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    a, b = x[..., first], x[..., second]
    y, off = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    most = (a.abs() + b.abs()) * abs(magnitude) * (angle_off + 4 * U)
    off[..., first], off[..., second] = most, most
    return y, off


def norm(x, w, eps):
    """(x / rms, 1 / rms, w in 64 bits)."""
    x = x.double().cpu()
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    return x * r, r, torch.ones(x.shape[-1], dtype=torch.float64) if w is None else w.double().cpu()


def norm_rotate(x, w, eps, rotary, positions):
    """(result, off): squares of d values in a tree below 16 deep, the root's inverse within 2 steps, two products: 24 u of the normed value."""
    n, _, w = norm(x, w, eps)
    y, off = turn(n * w, *_split(rotary, positions))
    _, spread = _absolute(n * w, rotary, positions)
    return y, off + 24 * U * spread


def norm_rotate_grad(g, x, w, eps, rotary, positions, terms):
    """(dx, its off, dw, its off); terms: summands of dw that one thread adds up one after the other."""
    n, r, w = norm(x, w, eps)
    gt, off = turn(g, *_split(rotary, positions), back=True)
    h, off_h = gt * w, off * w.abs()
    mean = (h * n).mean(-1, keepdim=True)
    dx = r * (h - n * mean)
    dx_off = r * (off_h + n.abs() * (off_h * n.abs()).mean(-1, keepdim=True) + 48 * U * (h.abs() + n.abs() * (h * n).abs().mean(-1, keepdim=True)))
    dw = (gt * n).sum((0, 1, 2))
    dw_off = (off * n.abs()).sum((0, 1, 2)) + (terms + 64) * U * (gt * n).abs().sum((0, 1, 2)) + U * dw.abs()
    return dx, dx_off, dw, dw_off


def _split(rotary, positions):
    if rotary is None:
        return torch.zeros(0), None, torch.zeros((1, 1), dtype=torch.int32), True, 1.0
    freq, axis, interleaved, magnitude = rotary
    return freq, axis, positions, interleaved, magnitude


def _absolute(x, rotary, positions):
    """Sum of a pair's magnitudes at both its channels (and the channel's own elsewhere), times the magnitude."""
    freq, axis, positions, interleaved, magnitude = _split(rotary, positions)
    n = len(freq)
    first = torch.arange(n) * (2 if interleaved else 1)
    second = first + (1 if interleaved else n)
    y = x.abs().clone()
    both = (y[..., first] + y[..., second]) * abs(magnitude)
    y[..., first], y[..., second] = both, both
    return x, y
