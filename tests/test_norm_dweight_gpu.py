"""dweight of the norm's backward pass within the rounding of its own chain of additions.

A thread adds up its CTA's rows, N / C of them for C CTAs; 32 lanes add up the C partials, C / 32 each, and a tree of five additions
the lanes.  Each product costs two roundings (xhat, and the fused multiply-add's is the addition's own).  C lies between 148 (or N)
and the rows of the workspace, and N / C + C / 32 is largest at one of the two; 3 more for the partial rows of either quotient.
Every addition is off by u = 2^-24 of the sum of magnitudes at most."""
import pytest
import torch

from oracle import step_oracle as S
from paper_2605_07244_b200 import binding as B

from test_rmsnorm_gpu import BF16, F32, MANY, U, _built, random_rows, run_bwd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,H", MANY + [(1, 64), (3, 4096), (147, 1024), (149, 1024), (593, 64), (60000, 64), (40000, 257), (1500, 16400)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_dweight_within_its_chain_of_additions(N, H, dtype):
    dy, h = random_rows(N, H, dtype, 1), random_rows(N, H, dtype, 2)
    w = torch.randn(H, generator=torch.Generator().manual_seed(7)).cuda()
    rstd = S.rmsnorm_residual_fwd(h, None, w, 0.0, 1e-6)[1].float().cuda()
    out = run_bwd(dy, None, h, w, rstd)
    _, want, _, mags = S.rmsnorm_residual_bwd(dy, None, h, w, 0.0, rstd)
    most = B.workspace_bytes(B.WS_RMSNORM_BWD, N, 0, H) // (4 * H)
    chain = max(N / c + c / 32 for c in (min(N, 148), min(N, most))) + 5 + 2 + 3
    err = (out["dw"].double().cpu() - want).abs()
    assert bool((err <= mags * chain * U + 1e-37).all()), float((err / (mags * chain * U + 1e-37)).max())
