"""A list of tensors holds addresses.  Where a parameter's own .grad was given, a call after autograd has made another one is refused
instead of stepping on the old one."""
import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

CALLS = [lambda ts: B.mrl_grad_norm(ts, 1.0), lambda ts: B.mrl_adamw_step(ts, B.AdamwParams(lr=1e-3, step=1, eps=1e-8))]


def slot(p, grad):
    n = p.numel()
    return B.TensorSlot(grad, p, None, torch.zeros(n, device=p.device), torch.zeros(n, device=p.device))


@pytest.mark.parametrize("call", CALLS)
def test_a_replaced_gradient_is_refused(call):
    p, q = (torch.nn.Parameter(torch.ones(8)) for _ in range(2))
    for t in (p, q):
        (2 * t).sum().backward()
    tensors = B.TensorList([slot(p, p.grad), slot(q, q.grad)])
    tensors.check("here")
    q.grad.zero_()                                   # the same tensor, other values
    (3 * q).sum().backward()
    tensors.check("here")
    q.grad = None
    with pytest.raises(B.MrlError, match="gradient"):
        call(tensors)
    (3 * q).sum().backward()
    with pytest.raises(B.MrlError, match="gradient"):
        call(tensors)
    B.TensorList([slot(p, p.grad), slot(q, q.grad)]).check("here")


def test_gradients_of_the_callers_own_are_not_looked_at():
    p = torch.nn.Parameter(torch.ones(8))
    own = torch.ones(8)
    lists = [B.TensorList([slot(p, own), B.TensorSlot(own), slot(2 * p, own)]), B.TensorList([slot(p.detach(), own)])]
    (2 * p).sum().backward()
    p.grad = None
    for tensors in lists:
        tensors.check("here")


@pytest.mark.gpu
def test_steps_on_gradients_made_anew():
    build.build()
    p = torch.nn.Parameter(torch.ones(300, device="cuda"))
    m, v = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    norm, ws = torch.empty(1, device="cuda"), torch.empty(B.workspace_bytes(B.WS_GRAD_NORM, 0, 0), dtype=torch.uint8, device="cuda")
    ap = B.AdamwParams(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8)
    q = torch.nn.Parameter(torch.ones(300, dtype=torch.float64))
    opt = torch.optim.AdamW([q], lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0)
    tensors = None
    for t in range(1, 5):
        for one in (p, q):
            one.grad = None
            ((t + torch.arange(300, device=one.device) % 7) * one).sum().backward()
        if tensors is not None:
            with pytest.raises(B.MrlError, match="gradient"):
                B.mrl_adamw_step(tensors, ap)
        tensors, ap.step = B.TensorList([B.TensorSlot(p.grad, p, None, m, v)]), t
        B.mrl_grad_norm(tensors, 0.0, norm, None, ws)
        B.mrl_adamw_step(tensors, ap)
        opt.step()
        assert abs(float(norm) - float(q.grad.norm())) <= 35 * 2.0 ** -24 * float(q.grad.norm())
        # each step: 24 u of an update of about lr, and 3 u of the parameter; the moments' errors (14 u) with it
        assert float((p.detach().double().cpu() - q.detach()).abs().max()) <= t * (40 * 1e-2 + 3) * 2.0 ** -24
