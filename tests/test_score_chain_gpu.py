"""Scoring a frozen model in 8 bits and learning from it, as one run: norm with e4m3 rows -> product -> top tokens -> distillation of
the learner's logits, directly, from a graph and on two streams."""
import pytest
import torch

from oracle import score_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

from test_top_gpu import HALF, chain

pytestmark = pytest.mark.gpu
N, H, V, TOP, T = 150, 384, 6001, 24, 1.5


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


class Run:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        e = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        self.x, self.gain = r(N, H).to(torch.bfloat16).cuda(), (1 + 0.1 * r(H)).cuda()
        self.W = (r(V, H) * 2 * H ** -0.5).to(torch.bfloat16).cuda()
        self.z = (2 * r(N, V)).to(torch.bfloat16).cuda()
        self.mask = (torch.rand(N, generator=g) < 0.9).to(torch.uint8).cuda()
        self.ids = torch.randint(0, V, (N,), generator=g, dtype=torch.int32).cuda()
        self.x8, self.xs, self.w8, self.ws = e(N, H, t=torch.uint8), e(N, 3), e(V, H, t=torch.uint8), e(-(-V // 128), 3)
        self.teacher, self.logp, self.entropy = e(N, V, t=torch.bfloat16), e(N), e(N)
        self.top_ids, self.top_logp = e(N, TOP, t=torch.int32), e(N, TOP)
        self.dz, self.kl, self.loss = e(N, V, t=torch.bfloat16), e(N), e(1)
        self.status, self.stats = e(1, t=torch.int32), e(2, t=torch.int64)
        self.work = torch.empty(B.workspace_bytes(B.WS_DISTILL, N, V), dtype=torch.uint8, device="cuda")
        self.np = B.NormParams(1e-6, 0.0, 128, 0)
        self.dp = B.DistillParams(T, 1.0, B.DISTILL_FORWARD, B.REST_EVENT, 1e-6, 0, 0.0)
        B.mrl_e4m3_quantize(self.W, self.w8, self.ws, 128)

    def step(self, stream=None):
        B.mrl_rmsnorm_residual_fwd(self.x, None, self.gain, self.np, y8=self.x8, scales=self.xs, stream=stream)
        B.mrl_e4m3_product(self.x8, self.xs, self.w8, self.ws, self.teacher, self.status, stream=stream)
        B.mrl_top_logprobs(self.teacher, self.ids, self.mask, T, self.logp, None, self.entropy, self.top_ids, self.top_logp, self.status,
                           stream=stream)
        B.mrl_distill_loss_fwd_bwd(self.z, self.top_ids, self.top_logp, self.mask, None, self.dp, self.dz, self.kl, self.loss, self.stats,
                                   self.status, self.work, stream=stream)


OUT = ("x8", "xs", "teacher", "logp", "entropy", "top_ids", "top_logp", "dz", "kl", "loss", "stats")


def test_the_chain_against_the_oracle():
    a = Run(1)
    a.step()
    torch.cuda.synchronize()
    assert int(a.status) == 0
    cpu = lambda t: t.cpu()  # noqa: E731
    want, size = S.product(cpu(a.x8).view(torch.float8_e4m3fn), cpu(a.xs), cpu(a.w8).view(torch.float8_e4m3fn), cpu(a.ws))
    # bf16 keeps eight bits: a rounding is off by half a step, 2^-8 of the value (values just above a power of two)
    assert bool(((cpu(a.teacher).double() - want).abs() <= 2.0 ** -8 * want.abs() + size * 12 * 2.0 ** -23).all())
    # e4m3 keeps three bits: each factor is off by at most 2^-4 of itself, their product by 2^-3 + 2^-8
    y = torch.nn.functional.rms_norm(a.x.double(), (H,), a.gain.double(), 1e-6).cpu()
    exact, bound = y @ a.W.double().cpu().T, y.abs() @ a.W.double().abs().cpu().T
    assert bool(((cpu(a.teacher).double() - exact).abs() <= bound * 0.14 + 0.01).all())
    on = cpu(a.mask).bool()
    _, logp, entropy, lists, top_logp = S.top_logprobs(cpu(a.teacher).float(), cpu(a.ids), T, TOP)
    assert torch.equal(cpu(a.top_ids).long()[on], lists[on]) and bool((cpu(a.top_ids)[~on] == -1).all())
    tol = chain(V) + 8 * HALF * 20
    assert float((cpu(a.logp).double() - logp)[on].abs().max()) <= tol and float((cpu(a.top_logp).double() - top_logp)[on].abs().max()) <= tol
    ref = S.distill_loss(cpu(a.z).float(), cpu(a.top_ids), cpu(a.top_logp), cpu(a.mask), None, T, 1.0, False, True, float(torch.tensor(1e-6)))
    assert a.stats.tolist() == [int(on.sum()), 0] and abs(float(a.loss) - ref["loss"]) <= 40 * tol * (1 + abs(ref["loss"]))
    off = (cpu(a.dz).double() - ref["dlogits"]).abs()
    assert bool((off <= 2.0 ** -8 * ref["dlogits"].abs() + 8 * tol * ref["parts"]).all())


def test_replayed_and_on_two_streams_bit_for_bit():
    a, b, pair = Run(2), Run(2), [Run(2), Run(3)]
    alone = Run(3)
    a.step()
    alone.step()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        b.step(side)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(2):
        graph.replay()
        for r, s in zip(pair, streams):
            r.step(s)
    torch.cuda.synchronize()
    for k in OUT:
        assert torch.equal(getattr(a, k), getattr(b, k)) and torch.equal(getattr(a, k), getattr(pair[0], k)), k
        assert torch.equal(getattr(alone, k), getattr(pair[1], k)), k
