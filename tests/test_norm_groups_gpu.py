"""The norm's 8-bit rows with every group of columns where calls of many rows run: CTAs that walk several rows, 8, 16 and 32
columns a thread, maxima that meet within a lane, within lanes and in shared memory, rows of whole granules and odd ones.
Tolerances: those of test_rmsnorm_gpu.py, whose check of codes is used."""
import pytest
import torch

from oracle import step_oracle as S
from paper_2605_07244_b200 import binding as B

from test_rmsnorm_gpu import BF16, F32, U, _built, chain, check_codes, random_rows, run_fwd  # noqa: F401

pytestmark = pytest.mark.gpu

# (rows, columns): 32 columns a thread from 2,049 rows of 2 to 16 KB on, 16 below and beyond, 8 for short rows; ragged last groups;
# odd rows
SHAPES = [(3000, 1024), (2100, 4096), (2100, 2056), (2100, 8192), (2500, 1027), (2100, 4095), (1900, 1544), (9000, 320), (450, 16384),
          (500, 16383)]


@pytest.mark.parametrize("N,H", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_group_where_calls_of_many_rows_run(N, H, dtype):
    x, res = random_rows(N, H, dtype, 1), random_rows(N, H, dtype, 2, scale=2.0)
    x[1::3] *= 0.03125                      # rows, and columns, of different size: a stale maximum would show
    res[:, H // 2:] *= 0.125
    w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
    some = torch.cat([torch.arange(40), torch.arange(N - 160, N)])
    y = S.rmsnorm_residual_fwd(x[some], res[some], w, 0.0, float(torch.tensor(1e-6, dtype=F32)))[2]
    rel = 2 * (chain(H) / 2 + 10) * U + 4 * U
    plain = run_fwd(x, res, w, want=("h", "y", "rstd"))
    for group in (0, 32, 64, 128, 256):
        out = run_fwd(x, res, w, group=group, want=("h", "y", "rstd", "q"))
        for k in ("h", "y", "rstd"):
            assert torch.equal(out[k], plain[k]), (group, k)
        check_codes(out["q"][some], out["scales"][some], y, group, rel, f"codes by {group}")
        # every row: each group's scale is its largest magnitude / 448, its largest code 448, within y's own rounding
        width = group or H
        wide = torch.nn.functional.pad(out["y"].float().abs(), (0, -H % width)).view(N, -1, width).amax(2)
        near = wide.double() / 448
        assert bool(((out["scales"].double() - near).abs() <= near * (torch.finfo(dtype).eps / 2 * (1 + 1e-3) + rel)).all()), group
        q = torch.nn.functional.pad(out["q"].view(torch.float8_e4m3fn).float().abs(), (0, -H % width)).view(N, -1, width).amax(2)
        assert bool((q == 448.0).all()), group
        again = run_fwd(x, res, w, group=group, want=("rstd", "q"))
        over_x, over_r = x.clone(), res.clone()
        over = run_fwd(over_x, over_r, w, group=group, want=("rstd", "q"), place={"h": over_r, "y": over_x})
        for one in (again, over):
            for k in ("q", "scales", "rstd"):
                assert torch.equal(one[k], out[k]), (group, k)
        assert torch.equal(over["h"], out["h"]) and torch.equal(over["y"], out["y"])
