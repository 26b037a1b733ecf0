"""The update of no elements (a rank whose shard is empty): the step counter and the status are those of any other call."""
import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

pytestmark = pytest.mark.gpu


def lists():
    e = lambda dtype=torch.float32: torch.empty(0, dtype=dtype, device="cuda")  # noqa: E731
    return [B.TensorList([]), B.TensorList([B.TensorSlot(e(), e(), None, e(), e()),
                                            B.TensorSlot(e(torch.bfloat16), e(torch.bfloat16), e(), e(), e())])]


@pytest.mark.parametrize("scale", [0.5, float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("counted", [False, True])
def test_status_and_counter_of_a_call_without_elements(scale, counted):
    build.build()
    finite = abs(scale) < float("inf")
    gs = torch.tensor([scale], device="cuda")
    for tensors in lists():
        for before in (0, B.DEV_BAD_TOKEN_ID):
            status = torch.tensor([before], dtype=torch.int32, device="cuda")
            count = torch.tensor([4], dtype=torch.int64, device="cuda")
            ws = torch.empty(B.workspace_bytes(B.WS_ADAMW, 0, 0), dtype=torch.uint8, device="cuda")
            ap = B.AdamwParams(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, step_dev=count.data_ptr() if counted else None)
            B.mrl_adamw_step(tensors, ap, gs, status, ws if counted else None)
            torch.cuda.synchronize()
            assert int(status) == (before if finite else before | B.DEV_NONFINITE_GRAD)
            assert int(count) == 4 + (counted and finite)
