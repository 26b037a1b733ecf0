"""The norm at the smallest eps that it takes, 2^-126, on rows whose squares leave float32's normal range.

A square is off by 2^-150 there and the mean by no more; against mean + eps >= 2^-126 that is u = 2^-24 relative, half of it in the
reciprocal root.  Otherwise the tolerances of test_rmsnorm_gpu.py; y in float32, so its half step is u."""
import pytest
import torch

from oracle import step_oracle as S
from paper_2605_07244_b200 import binding as B

from test_rmsnorm_gpu import F32, U, _built, chain, rows, run_fwd, within  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [1, 33, 1024, 4096, 16401])
def test_tiny_rows_at_the_smallest_eps(H):
    eps = 2.0 ** -126
    x = rows(7, H, F32, 1)
    for t, size in enumerate((1e-15, 1e-18, 1e-19, 1e-20, 1e-22, 1e-25, 1e-30)):
        x[t] *= size
    w = torch.ones(H, device="cuda")
    h, rstd, y = S.rmsnorm_residual_fwd(x, None, w, 0.0, eps)
    out = run_fwd(x, None, w, eps=eps, want=("y", "rstd"))
    rel = (chain(H) / 2 + 11) * U
    within(out["rstd"], rstd, rstd * rel, "rstd")
    within(out["y"], y, y.abs() * (U * (1 + 1e-3) + rel) + 1e-37, "y")
