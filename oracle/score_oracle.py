"""Plain CPU float64 oracle of scoring a frozen model in 8 bits and learning from its top tokens: e4m3 codes with block
scales and their product, the top tokens of a row of logits with its entropy, and the KL between a teacher's list and a
learner's logits with its gradient.

TEST INFRASTRUCTURE ONLY, like mrl_oracle: direct evaluation of the definitions, no code shared with the library.

Pins (tests/test_score_oracle_pins.py): autograd and central differences of the loss, hand values, brute-force sorting,
the KL of whole distributions, torch's e4m3 cast.
"""
from __future__ import annotations

import math

import torch

F64 = torch.float64
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
BLOCK = 128
NO_REST = -700.0        # ln p_r below which the learner gives the rest nothing, if it is masked:
MASK = -2.0 ** 26       # the largest of its logits is this or less


def _w(t):
    return torch.as_tensor(t).detach().cpu().to(F64)


def block_peaks(x, rows):
    """Largest magnitude of each block of rows x 128 elements; the last blocks may be short."""
    x = _w(x).abs()
    n, h = x.shape
    return torch.stack([torch.stack([x[a:a + rows, b:b + BLOCK].max() for b in range(0, h, BLOCK)]) for a in range(0, n, rows)])


def spread(scales, rows, n, h):
    """A block's scale at each of its elements."""
    return _w(scales).repeat_interleave(rows, 0)[:n].repeat_interleave(BLOCK, 1)[:, :h]


def product(x8, x_scales, w8, w_scales):
    """sum over columns of code * scale, and the sum of magnitudes its rounding errors go by."""
    x = _w(x8.float()) * spread(x_scales, 1, *x8.shape)
    w = _w(w8.float()) * spread(w_scales, BLOCK, *w8.shape)
    return x @ w.T, x.abs() @ w.abs().T


def top_logprobs(z, ids, temperature, top):
    """lse, logp, entropy and the top tokens of each row: the largest first, equal ones by their index; NaN is not listed."""
    z = _w(z)
    high = z.amax(1, keepdim=True)
    x = (z - high) / temperature            # (against the largest first: x - lse has no digits left where logits are 1e38)
    total = x.exp().sum(1, keepdim=True).log()
    lse, ln_p = (high / temperature + total)[:, 0], x - total
    entropy = -torch.where(ln_p == -math.inf, 0.0, ln_p.exp() * ln_p).sum(1)
    lists = torch.full((z.shape[0], top), -1, dtype=torch.int64)
    for t, row in enumerate(z.tolist()):
        best = sorted((v for v in range(len(row)) if row[v] == row[v]), key=lambda v: (-row[v], v))[:top]
        lists[t, :len(best)] = torch.tensor(best, dtype=torch.int64)
    top_logp = torch.where(lists >= 0, ln_p.gather(1, lists.clamp(min=0)), -math.inf)
    logp = None if ids is None else ln_p.gather(1, ids.long()[:, None])[:, 0]
    return lse, logp, entropy, lists, top_logp


def _xlogy(a, b):
    """a ln b, 0 where a = 0."""
    return 0.0 if a == 0.0 else (a * math.log(b) if b > 0.0 else -math.inf * a)


def distill_row(z, ids, logps, temperature, reverse, rest_event, floor):
    """KL and T dKL/dz of one row from its used places (ids, logps: lists), and the magnitudes the gradient is a difference of."""
    V = z.numel()
    x = z / temperature
    x = x - x.max()
    outside = torch.ones(V, dtype=torch.bool)
    outside[ids] = False
    total = x.exp().sum()
    p = x.exp() / total
    ln_p = x - total.log()
    ln_p_rest = float(torch.logsumexp(x[outside], 0) - total.log()) if bool(outside.any()) else -math.inf
    has_rest = ln_p_rest > -math.inf and not (ln_p_rest < NO_REST and float(z[outside].max()) <= MASK)
    p_rest = math.exp(ln_p_rest) if has_rest else 0.0
    within = torch.zeros(V, dtype=F64)                                      # softmax over the rest
    if has_rest:
        within[outside] = torch.softmax(x[outside], 0)
    l = torch.tensor(logps, dtype=F64)
    grad, parts = torch.zeros(V, dtype=F64), torch.zeros(V, dtype=F64)
    if not rest_event:
        l = l - torch.logsumexp(l, 0)
        q = l.exp()
        kl = float((q * (l - ln_p[ids])).sum())
        grad[ids], parts[ids] = p[ids] - q, p[ids] + q
        return kl, grad + p_rest * within, parts + p_rest * within
    q = l.exp()
    q_rest = max(1.0 - float(q.sum()), floor) if has_rest else 0.0
    if not reverse:
        mass = float(q.sum()) + q_rest
        kl = float((q * (l - ln_p[ids])).sum()) + (_xlogy(q_rest, q_rest) - q_rest * ln_p_rest if q_rest > 0 else 0.0)
        grad[ids], parts[ids] = mass * p[ids] - q, mass * p[ids] + q
        return kl, grad + (mass * p_rest - q_rest) * within, parts + (mass * p_rest + q_rest) * within
    pk, ratio = p[ids], ln_p[ids] - l
    terms = torch.where(pk > 0, pk * ratio, 0.0)
    ratio_rest = ln_p_rest - math.log(q_rest) if has_rest else 0.0
    kl = float(terms.sum()) + p_rest * ratio_rest
    size = float(terms.abs().sum()) + p_rest * abs(ratio_rest) + 1.0
    grad[ids], parts[ids] = torch.where(pk > 0, pk * (ratio - kl), 0.0), torch.where(pk > 0, pk * (ratio.abs() + size), 0.0)
    return kl, grad + p_rest * (ratio_rest - kl) * within, parts + p_rest * (abs(ratio_rest) + size) * within


def distill_loss(z, top_ids, top_logp, mask, weight, temperature=1.0, coeff=1.0, reverse=False, rest_event=True, floor=0.0,
                 denominator=0.0):
    """loss, row_kl, dlogits, the gradient's parts, the sum of the loss terms' magnitudes, and each row's state: 0 off, 1 valid, 2 refused."""
    z, top_logp = _w(z), _w(top_logp)
    N, V = z.shape
    state, used = [], []
    for t in range(N):
        places = [(int(i), float(l)) for i, l in zip(top_ids[t].tolist(), top_logp[t].tolist()) if i >= 0 and l != -math.inf]
        used.append(places)
        ids = [i for i, _ in places]
        if mask is not None and not int(mask[t]):
            state.append(0)
        elif any(i >= V for i in ids) or len(set(ids)) < len(ids) or any(not l < math.inf for _, l in places):
            state.append(2)
        else:
            state.append(1 if places else 0)
    d = denominator if denominator > 0 else float(state.count(1))
    row_kl, grad, parts, terms = torch.zeros(N, dtype=F64), torch.zeros(N, V, dtype=F64), torch.zeros(N, V, dtype=F64), [0.0]
    for t in range(N):
        if state[t] != 1:
            continue
        ids, l = [i for i, _ in used[t]], [v for _, v in used[t]]
        kl, g, m = distill_row(z[t], ids, l, temperature, reverse, rest_event, floor)
        w = 1.0 if weight is None else float(weight[t])
        row_kl[t] = kl
        if w != 0.0:
            c = coeff * w / d
            terms.append(c * kl)
            grad[t], parts[t] = g * (c / temperature), m * abs(c / temperature)
    return {"loss": math.fsum(terms) if all(map(math.isfinite, terms)) else sum(terms), "row_kl": row_kl, "dlogits": grad, "parts": parts,
            "size": sum(abs(x) for x in terms), "state": state}
