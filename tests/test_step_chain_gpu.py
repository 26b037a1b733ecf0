"""The last part of a learner's step as one run: norm -> fused LM head -> norm backward -> gradient norm -> AdamW, directly and
from a CUDA graph, against the same chain of oracles."""
import pytest
import torch

from oracle import mrl_oracle as O
from oracle import step_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

from helpers import make_lp, oracle_lp, rel_l2

pytestmark = pytest.mark.gpu

N, H, V, SEQ = 300, 256, 4000, 5
EPS = float(torch.tensor(1e-6))


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


class Learner:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        bf = lambda t: t.to(torch.bfloat16).cuda()  # noqa: E731
        self.x, self.res, self.dh = bf(r(N, H)), bf(2 * r(N, H)), bf(1e-3 * r(N, H))
        self.gain, self.W = (1 + 0.1 * r(H)).cuda(), bf(r(V, H) * (2.0 / H ** 0.5))
        self.ids = torch.randint(0, V, (N,), generator=g, dtype=torch.int32).cuda()
        self.cu = torch.tensor([0, 50, 120, 121, 200, N], dtype=torch.int32).cuda()
        self.adv = r(SEQ).cuda()
        e = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        f = torch.float32
        self.h, self.hidden, self.rstd = e(N, H), e(N, H), e(N, t=f)
        self.dHidden, self.dW, self.dx, self.dgain = e(N, H), e(V, H), e(N, H), e(H, t=f)
        self.logp, self.loss, self.status = e(N, t=f), e(2, t=f), e(1, t=torch.int32)
        self.norm, self.coef, self.count = e(1, t=f), e(1, t=f), e(1, t=torch.int64)
        blocks = V * H // B.STATE_BLOCK
        self.m, self.v = e(V * H, t=torch.uint8), e(V * H, t=torch.uint8)
        self.ms, self.vs, self.gm, self.gv = e(blocks, t=f), e(blocks, t=f), e(H, t=f), e(H, t=f)
        self.master = self.W.float().view(-1)
        ws = lambda *a: torch.empty(max(256, B.workspace_bytes(*a)), dtype=torch.uint8, device="cuda")  # noqa: E731
        self.w_head, self.w_norm = ws(B.WS_FUSED_LMHEAD, N, V, H, B.BF16, SEQ), ws(B.WS_RMSNORM_BWD, N, 0, H)
        self.w_sum, self.w_adam = ws(B.WS_GRAD_NORM, 0, 0), ws(B.WS_ADAMW, 0, 0)
        self.list = B.TensorList([
            B.TensorSlot(self.dW.view(-1), self.W.view(-1), self.master, self.m, self.v, self.ms, self.vs, 0.01),
            B.TensorSlot(self.dgain, self.gain, None, self.gm, self.gv, rng_first=V * H // 2)])
        self.ap = B.AdamwParams(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, seed=1, rounding=B.ROUND_SEEDED,
                                step_dev=self.count.data_ptr())
        self.np, self.lp = B.NormParams(EPS, 0.0, 0, 0), make_lp()

    def step(self, stream=None):
        B.mrl_rmsnorm_residual_fwd(self.x, self.res, self.gain, self.np, self.h, self.hidden, rstd=self.rstd, stream=stream)
        B.mrl_fused_lmhead_loss_fwd_bwd(self.hidden, self.W, self.ids, None, self.cu, self.adv, None, None, None, self.lp,
                                        self.dHidden, self.dW, self.logp, self.loss, None, self.status, self.w_head,
                                        stream=stream)
        B.mrl_rmsnorm_residual_bwd(self.dHidden, self.dh, self.h, self.gain, self.rstd, self.np, self.dx, self.dgain,
                                   self.w_norm, stream=stream)
        B.mrl_grad_norm(self.list, 0.01, self.norm, self.coef, self.w_sum, stream=stream)
        B.mrl_adamw_step(self.list, self.ap, self.coef, self.status, self.w_adam, stream=stream)


def test_one_step_against_the_chain_of_oracles():
    a = Learner(1)
    gain0, W0 = a.gain.clone(), a.W.clone()
    a.step()
    torch.cuda.synchronize()
    assert int(a.status) == 0 and int(a.count) == 1
    h, rstd, y = S.rmsnorm_residual_fwd(a.x, a.res, gain0, 0.0, EPS)
    assert rel_l2(a.hidden.cpu(), y) < 2.0 ** -8
    ref = O.fused_lmhead_loss(a.hidden.cpu(), W0.cpu(), a.ids.cpu(), None, a.cu.cpu(), a.adv.cpu(), None, None, None, oracle_lp(a.lp))
    assert rel_l2(a.dHidden.cpu(), ref["dHidden"]) < 1e-2 and rel_l2(a.dW.cpu(), ref["dW"]) < 1e-2
    dx, dgain, _, _ = S.rmsnorm_residual_bwd(a.dHidden, a.dh, a.h, gain0, 0.0, a.rstd)
    assert rel_l2(a.dx.cpu(), dx) < 2.0 ** -8 and rel_l2(a.dgain.cpu(), dgain) < 1e-5
    norm, coef = S.grad_norm([a.dW.cpu(), a.dgain.cpu()], float(torch.tensor(0.01)))
    assert coef < 1 and abs(float(a.norm) - norm) < 1e-5 * norm and abs(float(a.coef) - coef) < 1e-5 * coef
    zero = torch.zeros(H, dtype=torch.float64)
    want, _, _, _ = S.adamw(gain0, a.dgain, zero, zero, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, float(a.coef))
    assert float((a.gain.cpu().double() - want).abs().max()) < 1e-6
    zero = torch.zeros(V * H, dtype=torch.float64)
    want, _, _, _ = S.adamw(W0.view(-1), a.dW.view(-1), zero, zero, 1e-3, 0.9, 0.999, 1e-8, float(torch.tensor(0.01)), 1, float(a.coef))
    assert float((a.master.cpu().double() - want).abs().max()) < 1e-6
    assert torch.equal(a.W.view(-1), a.master.to(torch.bfloat16))


def test_steps_replayed_from_a_graph_are_the_direct_steps_bit_for_bit():
    a, b = Learner(2), Learner(2)
    warm = Learner(3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    warm.step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.step(side)
    for _ in range(3):
        a.step()
        graph.replay()
    torch.cuda.synchronize()
    assert int(a.count) == int(b.count) == 3
    for k in ("hidden", "h", "rstd", "dHidden", "dW", "dx", "dgain", "logp", "loss", "norm", "coef", "W", "master", "gain", "m", "v",
              "ms", "vs", "gm", "gv"):
        x, y = getattr(a, k), getattr(b, k)
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k


def test_two_learners_on_two_streams_with_workspaces_of_their_own():
    alone, pair = [Learner(4), Learner(5)], [Learner(4), Learner(5)]
    for a in alone:
        a.step()
        a.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(2):
        for a, s in zip(pair, streams):
            a.step(s)
    torch.cuda.synchronize()
    for a, b in zip(alone, pair):
        for k in ("dx", "dgain", "W", "m", "v", "gain", "norm"):
            assert torch.equal(getattr(a, k).view(torch.uint8), getattr(b, k).view(torch.uint8)), k
