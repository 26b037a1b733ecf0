"""Pins of oracle/score_oracle.py: autograd, differences, hand values, brute force."""
import math

import pytest
import torch

from oracle import score_oracle as S

F64 = torch.float64


def case(seed, V=11, K=4):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(3, V, generator=g, dtype=F64)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(3)])
    logq = torch.log_softmax(torch.randn(3, V, generator=g, dtype=F64), 1).gather(1, ids)
    return z, ids, logq


def autograd_loss(z, ids, logq, T, reverse, event):
    """From probabilities of whole events, differentiated by torch."""
    p = torch.softmax(z / T, 1)
    pk, q = p.gather(1, ids), logq.exp()
    if event:
        pk, q = torch.cat([pk, 1 - pk.sum(1, keepdim=True)], 1), torch.cat([q, 1 - q.sum(1, keepdim=True)], 1)
    else:
        q = q / q.sum(1, keepdim=True)
    a, b = (pk, q) if reverse else (q, pk)
    return (a * (a / b).log()).sum(1)


@pytest.mark.parametrize("reverse,event", [(False, True), (True, True), (False, False)])
@pytest.mark.parametrize("T", [1.0, 0.7, 2.0])
def test_gradient_is_that_of_autograd_and_of_differences(reverse, event, T):
    z, ids, logq = case(1)
    w = torch.tensor([0.5, 2.0, 1.0], dtype=F64)
    out = S.distill_loss(z, ids, logq, None, w, T, 0.3, reverse, event)
    x = z.clone().requires_grad_()
    kl = autograd_loss(x, ids, logq, T, reverse, event)
    loss = 0.3 * (w * kl).sum() / 3
    loss.backward()
    assert torch.allclose(out["row_kl"], kl.detach(), atol=1e-12) and abs(out["loss"] - float(loss)) < 1e-12
    assert torch.allclose(out["dlogits"], x.grad, atol=1e-12)
    h = 1e-5
    for v in range(z.shape[1]):
        up, down = z.clone(), z.clone()
        up[1, v] += h
        down[1, v] -= h
        d = (S.distill_loss(up, ids, logq, None, w, T, 0.3, reverse, event)["loss"] -
             S.distill_loss(down, ids, logq, None, w, T, 0.3, reverse, event)["loss"]) / (2 * h)
        assert abs(d - float(out["dlogits"][1, v])) < 1e-9


@pytest.mark.parametrize("reverse", [False, True])
def test_own_list_has_no_loss_and_no_gradient(reverse):
    z, ids, _ = case(2)
    logq = torch.log_softmax(z, 1).gather(1, ids)
    out = S.distill_loss(z, ids, logq, None, None, reverse=reverse, floor=1e-30)
    assert out["row_kl"].abs().max() < 1e-12 and out["dlogits"].abs().max() < 1e-12


def test_whole_vocabulary_is_the_whole_kl():
    z, _, _ = case(3, V=5)
    logq = torch.log_softmax(torch.tensor([[0.1, 2.0, -1.0, 0.0, 0.5]], dtype=F64), 1).expand(3, 5)
    ids = torch.arange(5).expand(3, 5)
    kl = torch.nn.functional.kl_div(torch.log_softmax(z, 1), logq, log_target=True, reduction="none").sum(1)
    assert torch.allclose(S.distill_loss(z, ids, logq, None, None)["row_kl"], kl, atol=1e-12)
    back = torch.nn.functional.kl_div(logq, torch.log_softmax(z, 1), log_target=True, reduction="none").sum(1)
    assert torch.allclose(S.distill_loss(z, ids, logq, None, None, reverse=True, floor=1e-9)["row_kl"], back, atol=1e-12)


def test_hand_value():
    z = torch.tensor([[0.0, 0.0, 0.0, 0.0]], dtype=F64)
    out = S.distill_loss(z, torch.tensor([[2, -1]]), torch.tensor([[math.log(0.5), 0.0]], dtype=F64), None, None)
    assert abs(out["loss"] - (0.5 * math.log(2.0) + 0.5 * math.log(0.5 / 0.75))) < 1e-12
    assert torch.allclose(out["dlogits"][0], torch.tensor([1, 1, -3, 1], dtype=F64) / 12, atol=1e-12)


def test_gradient_rows_sum_to_zero_and_states():
    z, ids, logq = case(4)
    for reverse, event in ((False, True), (True, True), (False, False)):
        g = S.distill_loss(z, ids, logq, None, None, reverse=reverse, rest_event=event, floor=1e-9)["dlogits"]
        assert g.sum(1).abs().max() < 1e-12
    ids = torch.tensor([[1, 1], [0, 11], [-1, -5]])
    lq = torch.tensor([[-1.0, -1.0], [-1.0, -1.0], [-1.0, -1.0]])
    assert S.distill_loss(z, ids, lq, None, None)["state"] == [2, 2, 0]
    assert S.distill_loss(z, ids, lq, torch.tensor([0, 1, 1]), None)["state"] == [0, 2, 0]
    lq = torch.tensor([[math.nan, -math.inf], [math.inf, -1.0], [-1.0, -1.0]])
    assert S.distill_loss(z, torch.tensor([[1, 2], [1, 2], [1, 2]]), lq, None, None)["state"] == [2, 2, 1]


def test_top_tokens_by_brute_force_and_uniform_rows():
    z = torch.tensor([[1.0, 3.0, 3.0, -math.inf, math.nan], [0.0, -0.0, 0.0, -1.0, 0.0]], dtype=F64)
    _, _, _, ids, _ = S.top_logprobs(z, None, 1.0, 5)
    assert ids.tolist() == [[1, 2, 0, 3, -1], [0, 1, 2, 4, 3]]
    lse, logp, entropy, ids, top = S.top_logprobs(torch.zeros(1, 7), torch.tensor([3]), 0.5, 2)
    ln7 = math.log(7)
    assert abs(float(lse) - ln7) < 1e-12 and abs(float(logp) + ln7) < 1e-12 and abs(float(entropy) - ln7) < 1e-12
    assert ids.tolist() == [[0, 1]] and torch.allclose(top, torch.full((1, 2), -ln7, dtype=F64))
    x = torch.randn(4, 9, generator=torch.Generator().manual_seed(0), dtype=F64)
    p = torch.softmax(x / 2.0, 1)
    assert torch.allclose(S.top_logprobs(x, None, 2.0, 1)[2], -(p * p.log()).sum(1), atol=1e-12)


def test_blocks_and_product():
    x = torch.arange(300.0)[None] * torch.tensor([[1.0], [-2.0], [3.0]])
    assert S.block_peaks(x, 1).tolist() == [[127.0, 255.0, 299.0], [254.0, 510.0, 598.0], [381.0, 765.0, 897.0]]
    assert S.block_peaks(x, 128).tolist() == [[381.0, 765.0, 897.0]]
    a, b = torch.tensor([[1.0, 2.0]]).to(torch.float8_e4m3fn), torch.tensor([[0.5, -3.0], [1.0, 1.0]]).to(torch.float8_e4m3fn)
    out, size = S.product(a, torch.tensor([[2.0]]), b, torch.tensor([[10.0]]))
    assert out.tolist() == [[-110.0, 60.0]] and size.tolist() == [[130.0, 60.0]]
