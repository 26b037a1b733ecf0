"""The distillation with a workspace of exactly the places that its lists have."""
import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

import test_distill_gpu as D

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", sorted(D.KINDS))
@pytest.mark.parametrize("N,V,top", [(1, 1, 1), (3, 700, 1), (9, 3001, 7), (301, 1003, 33), (600, 2000, 64), (5, 70001, 127)])
def test_a_workspace_for_these_places_is_enough(N, V, top, kind):
    build.build()
    z, flat = D.rows(N, V, torch.float32, N + V)
    ids, logq = D.lists(z, top, 2, unused=False)
    dp = D.params(kind)
    want = D.run(z, flat, ids, logq, None, None, dp)         # (a workspace for the longest lists)
    n = B.workspace_bytes(B.WS_DISTILL, N, V, 0, B.F32, top)
    assert n <= B.workspace_bytes(B.WS_DISTILL, N, V)
    room = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    zd, dz = z.cuda().contiguous(), torch.empty(N, V, device="cuda")
    kl, loss = torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    B.mrl_distill_loss_fwd_bwd(zd, ids.cuda(), logq.cuda(), None, None, dp, dz, kl, loss, None, None, room[:n])
    torch.cuda.synchronize()
    assert bool((room[n:] == 0xA5).all())
    assert torch.equal(kl.cpu(), want["row_kl"]) and float(loss) == want["loss"]
    D.check(z, {**want, "dz": dz.cpu()}, ids, logq, None, None, dp)
    with pytest.raises(B.MrlError):
        B.mrl_distill_loss_fwd_bwd(zd, ids.cuda(), logq.cuda(), None, None, dp, dz, kl, loss, None, None, room[:n - 1])
