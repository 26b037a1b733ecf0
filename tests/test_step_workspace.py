"""Workspaces that are smaller than their element count says (expanded or strided tensors) are refused before a launch."""
import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

BAD = [lambda d: torch.zeros(1, dtype=torch.uint8, device=d).expand(1 << 20),
       lambda d: torch.zeros(1024, 1, dtype=torch.uint8, device=d).expand(1024, 1024),
       lambda d: torch.zeros(1 << 12, dtype=torch.uint8, device=d)[::2]]


@pytest.mark.parametrize("make", BAD)
def test_a_workspace_has_to_be_contiguous(make):
    with pytest.raises(B.MrlError):
        B._workspace(make("cpu"), -1, "here")
    whole = torch.zeros(1 << 12, dtype=torch.uint8)
    assert B._workspace(whole, -1, "here") == (whole.data_ptr(), 1 << 12) and B._workspace(None, -1, "here") == (None, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("make", BAD)
def test_the_entry_points_refuse_it(make):
    build.build()
    ws = make("cuda")
    x, w, r = torch.ones(4, 64, device="cuda"), torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    tensors = B.TensorList([B.TensorSlot(w.clone(), w.clone(), None, w.clone(), w.clone())])
    with pytest.raises(B.MrlError):
        B.mrl_rmsnorm_residual_bwd(x, None, x, w, r, B.NormParams(1e-6, 0.0, 0, 0), x.clone(), w.clone(), ws)
    with pytest.raises(B.MrlError):
        B.mrl_grad_norm(tensors, 1.0, r[:1], None, ws)
    with pytest.raises(B.MrlError):
        B.mrl_adamw_step(tensors, B.AdamwParams(lr=1e-3, eps=1e-8, step_dev=count.data_ptr()), workspace=ws)
    torch.cuda.synchronize()
    assert int(count) == 0 and bool((r == 1).all())
