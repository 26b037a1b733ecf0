"""A rest that the learner leaves next to nothing: without masks it is an event like any other, however small (low temperatures); where it is masked there is none.

The definition here is written with torch and differentiated by it, apart from the oracle, and drops nothing by the size of a probability."""
import math

import pytest
import torch

from oracle import score_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

import test_distill_gpu as D

KINDS = sorted(D.KINDS)


def definition(z, ids, logq, T, kind, floor, rest=True):
    """KL of each row and its gradient, with or without the rest as an event (in the learner and the teacher)."""
    z = z.double().requires_grad_()
    ln_p = torch.log_softmax(z / T, 1)
    outside = torch.zeros_like(ln_p).scatter(1, ids.long(), -math.inf)
    mine, theirs = ln_p.gather(1, ids.long()), logq.double()
    q = theirs.exp()
    if kind == "none":
        share = q / q.sum(1, keepdim=True)
        kl = (share * (share.log() - mine)).sum(1)
    else:
        kl = (mine.exp() * (mine - theirs)).sum(1) if kind == "reverse" else (q * (theirs - mine)).sum(1)
        if rest:
            q_rest, ln_rest = (1 - q.sum(1)).clamp(min=floor), torch.logsumexp(ln_p + outside, 1)
            kl = kl + (ln_rest.exp() * (ln_rest - q_rest.log()) if kind == "reverse" else q_rest * (q_rest.log() - ln_rest))
    return kl.detach(), torch.autograd.grad(kl.sum(), z)[0]


def cold_rows(N, V, dtype, seed):
    """Unmasked logits: plain rows, rows with a listed token 9 above, with another one 9 above, and listed tokens 12 below."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(N, V, generator=g)
    ids = torch.stack([torch.randperm(V, generator=g)[:8] for _ in range(N)]).int()
    for t in range(N):
        if t % 4 == 1:
            z[t, int(ids[t, 3])] = 9.0 + z[t].max()
        elif t % 4 == 2:
            z[t, next(v for v in range(V) if v not in ids[t].tolist())] = 9.0 + z[t].max()
        elif t % 4 == 3:
            z[t, ids[t].long()] = -12.0
    logq = torch.log_softmax(torch.randn(N, 9, generator=g), 1)[:, :8].contiguous()
    return z.to(dtype), ids, logq


def same_as_definition(ref, z, ids, logq, T, kind, N, rest=True):
    kl, grad = definition(z, ids, logq, T, kind, D.FLOOR, rest)
    assert torch.allclose(ref["row_kl"], kl, rtol=1e-9, atol=1e-12)
    assert bool(((ref["dlogits"] - grad / N).abs() <= 1e-9 * (ref["parts"] + (grad / N).abs()) + 1e-30).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [0.01, 1e-3, 1e-6])
def test_oracle_at_low_temperatures(T, kind):
    z, ids, logq = cold_rows(12, 50, torch.float32, 1)
    ref = S.distill_loss(z, ids, logq, None, None, T, 1.0, kind == "reverse", kind != "none", D.FLOOR)
    same_as_definition(ref, z, ids, logq, T, kind, 12)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("mask,T,rest", [(-1e8, 1.0, False), (-2.0 ** 26, 1.0, False), (-1e30, 0.01, False), (-6.6e7, 1.0, True), (-1e4, 1.0, True),
                                         (-1e8, 1e6, True)])
def test_oracle_with_masks(mask, T, rest, kind):
    z, ids, logq = cold_rows(4, 50, torch.float32, 2)
    free = torch.ones(4, 50, dtype=torch.bool).scatter(1, ids.long(), False)
    z[free] = mask
    ref = S.distill_loss(z, ids, logq, None, None, T, 1.0, kind == "reverse", kind != "none", D.FLOOR)
    same_as_definition(ref, z, ids, logq, T, kind, 4, rest)


def check(z, got, ids, logq, dp):
    """As test_distill_gpu.check but for the smallest gradients: powers 2^t below 2^-126 are 0 in the kernel, and the factor of the softmax over the rest, 1 / (D T) at most
    where coeff = 1, is above 1 at low temperatures.  So an element can be off by 2^-126 / (D T) where that is more than the type's smallest normal number."""
    ref = S.distill_loss(z.float(), ids, logq, None, None, dp.temperature, dp.coeff, dp.direction == B.DISTILL_REVERSE, dp.rest == B.REST_EVENT, D.FLOOR)
    D.check(z, {**got, "dz": None}, ids, logq, None, None, dp)
    slack = D.kl_slack(z, ids, logq, dp.temperature, D.FLOOR)[:, None] if dp.direction == B.DISTILL_REVERSE else 1.0
    tol = (torch.finfo(z.dtype).eps / 2 * ref["dlogits"].abs() + 4 * (D.chain(z.shape[1]) + 8 * D.HALF) * slack * ref["parts"] +
           2.0 ** -126 * max(1.0, 1.0 / (len(z) * dp.temperature)))
    off = (got["dz"].double() - ref["dlogits"]).abs()
    assert bool((off <= tol).all()), float((off - tol).max())
    return ref


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,shift", [(0.01, 0.0), (1e-3, 0.0), (1e-6, 0.0), (1e-6, -2000.0), (1e-6, 2000.0)])
@pytest.mark.parametrize("N,V", [(420, 1003), (12, 40001)])
def test_low_temperatures(N, V, T, shift, kind, dtype):
    build.build()
    z, ids, logq = cold_rows(N, V, torch.float32, N)
    z = (z + shift).to(dtype)
    T = float(torch.tensor(T))
    dp = D.params(kind, T)
    got = D.run(z, z.reshape(-1), ids, logq, None, None, dp)
    assert got["status"] == 0 and got["dz"].isfinite().all()
    ref = check(z, got, ids, logq, dp)
    same_as_definition(ref, z, ids, logq, T, kind, N)
    again = D.run(z, z.reshape(-1), ids, logq, None, None, dp, in_place=True)
    assert torch.equal(got["dz"].view(torch.uint8), again["dz"].view(torch.uint8)) and torch.equal(got["row_kl"], again["row_kl"])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("mask,T", [(-1e8, 1.0), (-2.0 ** 26, 1.0), (-1e30, 0.01), (-6.6e7, 1.0), (-1e4, 1.0), (-1e8, 1e6), (-3e4, 0.001)])
@pytest.mark.parametrize("N,V", [(420, 1003), (8, 40001)])
def test_masks(N, V, mask, T, kind):
    build.build()
    z, ids, logq = cold_rows(N, V, torch.float32, 2)
    free = torch.ones(N, V, dtype=torch.bool).scatter(1, ids.long(), False)
    z[free] = mask
    T = float(torch.tensor(T))
    dp = D.params(kind, T)
    got = D.run(z, z.reshape(-1), ids, logq, None, None, dp)
    check(z, got, ids, logq, dp)
