"""Plain CPU float64 oracle of what stands around the loss pass in a learner's optimisation step: the root-mean-square
norm with the residual's addition in front of the LM head and its gradients, the norm of the step's gradients with the
clip factor, and the AdamW update (App. A: clipping at 1.0, AdamW) with states in 32 or 8 bits.

TEST INFRASTRUCTURE ONLY, like mrl_oracle: direct evaluation of the definitions, no code shared with the library.
Results are unrounded; what is stored in fewer bits is described by its position on the grid of representable values
(`grid`, `grid_target`), so that a test can say which of two neighbours a rounding may give.

Pins (tests/test_step_oracle_pins.py): autograd of the formula in float64, scale invariance, torch.optim.AdamW in float64,
the sign step of the first update, torch's e4m3 cast, the mean over all dithers, SplitMix64's published outputs.
"""
from __future__ import annotations

import torch

F64 = torch.float64
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
STATE_BLOCK = 256


def _w(t):
    return torch.as_tensor(t).detach().cpu().to(F64)


def rmsnorm_residual_fwd(x, residual, weight, offset, eps):
    """h = x + residual, rstd = 1 / sqrt(mean h^2 + eps), y = h rstd (weight + offset)."""
    h = _w(x) if residual is None else _w(x) + _w(residual)
    rstd = 1.0 / torch.sqrt((h * h).mean(dim=1) + eps)
    return h, rstd, h * rstd[:, None] * (_w(weight) + offset)


def group_scales(y, group):
    """max |y| / 448 of each group of columns (0: of the row), not below 2^-126; and the same for each column."""
    N, H = y.shape
    which = torch.arange(H) // (group if group else H)
    scales = torch.stack([y[:, which == k].abs().amax(dim=1) for k in range(int(which[-1]) + 1)], dim=1) / E4M3_MAX
    scales = scales.clamp_min(SCALE_MIN)
    return scales, scales[:, which]


def rmsnorm_residual_bwd(dy, dh, h, weight, offset, rstd):
    """Gradients from the stored h and rstd: dx, dweight, and the sums of magnitudes their rounding errors go by."""
    dy, h, r = _w(dy), _w(h), _w(rstd)[:, None]
    w = _w(weight) + offset
    xhat = h * r
    g = dy * w
    dx = r * (g - xhat * (g * xhat).mean(dim=1, keepdim=True))
    parts = r.abs() * (g.abs() + xhat.abs() * (g * xhat).abs().mean(dim=1, keepdim=True))
    if dh is not None:
        dx, parts = dx + _w(dh), parts + _w(dh).abs()
    return dx, (dy * xhat).sum(dim=0), parts, (dy * xhat).abs().sum(dim=0)


def grad_norm(grads, max_norm):
    total = sum((float((_w(g) ** 2).sum()) for g in grads), 0.0) ** 0.5
    return total, (max_norm / max(total, max_norm) if max_norm > 0 else 1.0)


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step, scale=1.0):
    """One step from float64 values; returns p, m, v, and the update without the decay."""
    g = _w(g) * scale
    m = beta1 * _w(m) + (1.0 - beta1) * g
    v = beta2 * _w(v) + (1.0 - beta2) * g * g
    update = (m / (1.0 - beta1 ** step)) / (torch.sqrt(v / (1.0 - beta2 ** step)) + eps)
    p = _w(p)
    return p - lr * (weight_decay * p + update), m, v, update


def block_scales(s):
    """max |s| / 448 over each STATE_BLOCK elements, not below 2^-126, repeated for each element."""
    n = s.numel()
    out = torch.stack([b.abs().max() for b in s.split(STATE_BLOCK)]) if n else torch.zeros(0, dtype=F64)
    out = (out / E4M3_MAX).clamp_min(SCALE_MIN)
    return out, out.repeat_interleave(STATE_BLOCK)[:n]


def e4m3_values():
    """The 256 e4m3 codes by definition: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    out = []
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        v = float("nan") if (c & 0x7F) == 0x7F else v
        out.append(-v if c & 0x80 else v)
    return torch.tensor(out, dtype=F64)


def e4m3_grid(a):
    """Distance between e4m3 values at magnitude a."""
    e = torch.floor(torch.log2(a.clamp_min(2.0 ** -60)))
    return torch.exp2(e.clamp_min(-6.0) - 3.0)


def bf16_grid(a):
    e = torch.floor(torch.log2(a.clamp_min(2.0 ** -126)))
    return torch.exp2(e.clamp_min(-126.0) - 7.0)


def grid_target(a, step, dither=None, top=None):
    """Magnitude a on a grid of `step`: the value it is rounded to (to nearest even, or down after the addition of
    dither / 65536 steps) and how far, in steps, it is from being rounded otherwise."""
    pos = a / step
    if dither is None:
        to = torch.round(pos)                                   # ties to even
        border = ((pos - torch.floor(pos)) - 0.5).abs()
    else:
        q = pos + _w(dither) / 65536.0
        to = torch.floor(q)
        border = torch.minimum(q - to, to + 1 - q)
    to = to * step
    return (to if top is None else to.clamp_max(top)), border


def splitmix64(x):
    mask = (1 << 64) - 1
    x = (x + 0x9E3779B97F4A7C15) & mask
    z = x
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
    return z ^ (z >> 31)


def dithers(n, seed, step, rng_first):
    """16 bits for m, v and the parameter of each of n elements."""
    key = splitmix64((splitmix64(seed) + step) & ((1 << 64) - 1))
    rm, rv, rp = [], [], []
    for i in range(n):
        w = splitmix64((key + rng_first + i // 2) & ((1 << 64) - 1)) >> (32 * (i % 2))
        rm.append(w & 0xFFFF)
        rv.append((w >> 16) & 0xFFFF)
        rp.append(int(format(rm[-1], "016b")[::-1], 2))
    return tuple(torch.tensor(t, dtype=torch.int64) for t in (rm, rv, rp))
