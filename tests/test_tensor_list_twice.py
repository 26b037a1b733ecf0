"""A parameter that is in the list twice (tied weights, say) would be updated by two CTAs at once: refused when the list is built."""
import pytest
import torch

from paper_2605_07244_b200 import binding as B


def slot(p, grad=None):
    n = p.numel()
    return B.TensorSlot(torch.ones(n) if grad is None else grad, p, None, torch.zeros(n), torch.zeros(n))


def test_a_parameter_may_be_in_a_list_once():
    p, q, none = torch.ones(8, 4), torch.ones(8), torch.empty(0)
    shared = torch.ones(32)
    B.TensorList([slot(p), slot(q), slot(none), slot(none), slot(torch.ones(32), shared), slot(torch.ones(32), shared)])
    B.TensorList([B.TensorSlot(shared), B.TensorSlot(shared)])          # gradients alone are only read
    for twice in ([slot(p), slot(q), slot(p)], [slot(p), slot(p.view(-1))], [slot(p), slot(p[:2])]):
        with pytest.raises(B.MrlError):
            B.TensorList(twice)
