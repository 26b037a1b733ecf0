"""Log-probs, policy loss and entropy with finite masks of any size in the logits: what a mask adds to a row is 0, in whichever thread or CTA it lies.

(z log2 e is rounded where it is a running maximum and not where it is subtracted from: in stretches of masks alone the powers of two are infinite or 0.)"""
import pytest
import torch

from oracle import mrl_oracle as O
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

from helpers import LOGP_ATOL, compare_policy_loss, dev, make_lp, oracle_lp, run_gpu_policy_loss
from test_entropy_gpu import ENT_ATOL, run as run_entropy

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def masked(V, dtype, pad):
    """For masks from -1e9 to the type's lowest value: the vocabulary's end, its first token, its last one, every other stretch of 3,000, all but every 97th token."""
    g = torch.Generator().manual_seed(V)
    v, out = torch.arange(V), []
    for fill in (-1e9, -1e10, -1e30, -3e37, torch.finfo(dtype).min):
        for where in (v >= V - V // 5, v == 0, v == V - 1, v // 3000 % 2 == 1, v % 97 != 5):
            z = torch.randn(V, generator=g) * 2.0
            z[where] = fill
            out.append(torch.cat([z, torch.zeros(pad)]))
    z = torch.stack(out).to(dtype)
    ids = torch.stack([torch.nonzero(r[:V] > -100)[int(torch.randint(0, 10, (1,), generator=g))][0] for r in z.float()]).int()
    return z, ids


SHAPES = [(1000, torch.bfloat16, 3), (1024, torch.float32, 0), (4096, torch.bfloat16, 0), (20008, torch.float32, 0), (40008, torch.bfloat16, 0), (151936, torch.bfloat16, 0),
          (262160, torch.bfloat16, 0), (128256, torch.float32, 0), (5003, torch.float32, 1)]


@pytest.mark.parametrize("V,dtype,pad", SHAPES)
def test_log_probs(V, dtype, pad):
    z, ids = masked(V, dtype, pad)
    logp, lse = torch.empty(len(z), device="cuda"), torch.empty(len(z), device="cuda")
    B.mrl_token_logprobs(dev(z), dev(ids), None, logp, lse, V=V)
    torch.cuda.synchronize()
    want, want_lse, _ = O.token_logprobs(z[:, :V], ids, None)
    assert logp.isfinite().all() and (logp.cpu().double() - want).abs().max() <= LOGP_ATOL
    assert (lse.cpu().double() - want_lse).abs().max() <= LOGP_ATOL


@pytest.mark.parametrize("V,dtype,pad", SHAPES)
def test_policy_loss(V, dtype, pad):
    z, ids = masked(V, dtype, pad)
    cu, adv = torch.tensor([0, 7, len(z)], dtype=torch.int32), torch.tensor([0.7, -1.1])
    lp = make_lp()
    ref = O.policy_loss(z[:, :V], ids, None, cu, adv, None, None, None, oracle_lp(lp))
    compare_policy_loss(run_gpu_policy_loss(z, ids, None, cu, adv, None, None, None, lp, V=V), ref, V, dtype, cancelling=True)


@pytest.mark.parametrize("ratio_level", [B.RATIO_TOKEN, B.RATIO_SEQUENCE])
@pytest.mark.parametrize("V,dtype,pad", SHAPES)
def test_entropy(V, dtype, pad, ratio_level):
    z, ids = masked(V, dtype, pad)
    cu, adv = torch.tensor([0, 7, len(z)], dtype=torch.int32), torch.tensor([0.7, -1.1])
    ent, logp = run_entropy(z, ids, None, cu, adv, V, ratio_level)
    assert (ent.double() - O.token_entropy(z[:, :V], ids, None)).abs().max() <= ENT_ATOL
    assert (logp.double() - O.token_logprobs(z[:, :V], ids, None)[0]).abs().max() <= LOGP_ATOL


def test_not_finite_rows_stay_so():
    z = torch.randn(3, 151936, dtype=torch.bfloat16)
    z[0, 5], z[1, 150000], z[2, 7] = float("nan"), float("nan"), float("inf")
    z[:2, :4000] = -1e30
    z[0, 5] = float("nan")
    logp = torch.zeros(3, device="cuda")
    B.mrl_token_logprobs(dev(z), torch.full((3,), 9000, dtype=torch.int32, device="cuda"), None, logp)
    assert logp.isnan().all()
