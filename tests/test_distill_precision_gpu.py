"""The distillation's gradient of long float32 rows, within the roundings of the order in which a row is summed (test_distill_gpu's `chain` allows for any order).

One CTA a row, 480 threads: a thread adds 16 pairs of a group to a sum of their own, that to its total, ten groups of 151,936 floats; 14 more additions join the block:
41 half steps (2^-24).  Each group may raise the maximum, a factor off by 2^-22 and a product: 5 half steps, ten times.  A term is off by 2^-22 of the power and by half
a step of its exponent t, |t| < 44 where logits are within 30 of the largest: 4 + 44 ln 2 < 35 half steps.  So the sum s is off by less than 41 + 50 + 35 = 126, and an
element 2^t p_r / s, p_r itself of s, by less than 35 + 2 * 126 + 13 more products and quotients = 300 half steps of the parts that the gradient is a difference of.  In
the reverse direction it is p (ln p - ln q - KL): as much again, for the logarithms and the KL, of parts with their sizes."""
import pytest
import torch

from oracle import score_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

import test_distill_gpu as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", sorted(D.KINDS))
@pytest.mark.parametrize("T", [1.0, 0.7])
def test_gradient_of_long_rows(T, kind):
    build.build()
    N, V, some = 300, 151936, 6
    T = float(torch.tensor(T))
    z, _ = D.rows(N, V, torch.float32, 11)
    ids, logq = D.lists(z[:some], 64, 5, T, unused=False)
    zd = z.cuda().contiguous()
    idsd, logqd = ids.cuda().repeat(N // some, 1), logq.cuda().repeat(N // some, 1)
    dz, kl, loss = torch.empty_like(zd), torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(B.workspace_bytes(B.WS_DISTILL, N, V, 0, B.F32, 64), dtype=torch.uint8, device="cuda")
    B.mrl_distill_loss_fwd_bwd(zd, idsd, logqd, None, None, D.params(kind, T, denominator=1.0), dz, kl, loss, None, None, ws)
    ref = S.distill_loss(z[:some], ids, logq, None, None, T, 1.0, kind == "reverse", kind != "none", D.FLOOR, 1.0)
    off = (dz[:some].cpu().double() - ref["dlogits"]).abs()
    tol = D.HALF * ref["dlogits"].abs() + (600 if kind == "reverse" else 300) * D.HALF * ref["parts"] + 2.0 ** -126 / T
    assert float((z[:some].amax(1) - z[:some].amin(1)).max()) < 30 * T
    assert bool((off <= tol).all()), float((off / tol).max())
