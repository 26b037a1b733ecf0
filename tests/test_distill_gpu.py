"""mrl_distill_loss_fwd_bwd against the float64 oracle.

The sum over the rest carries an error of `chain` (test_top_gpu.py derives it); ln p and with it every probability inherits it.  A gradient is
a difference of magnitudes `parts`, each off by that much, and rounded once; a row's KL moves by at most chain times 1 + the largest
|ln p - ln q| of its terms, which `kl_slack` takes from the row, and is rounded once."""
import math

import pytest
import torch

from oracle import score_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

from test_top_gpu import HALF, chain, rows

pytestmark = pytest.mark.gpu
KINDS = {"forward": (B.DISTILL_FORWARD, B.REST_EVENT), "reverse": (B.DISTILL_REVERSE, B.REST_EVENT), "none": (B.DISTILL_FORWARD, B.REST_NONE)}
FLOOR = 2.0 ** -20


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def lists(z, top, seed, T=1.0, noise=1.0, unused=True):
    """A teacher near the learner: its top tokens with log-probs at T, some places unused (-1 or -inf)."""
    g = torch.Generator().manual_seed(seed)
    t = (z.float().clamp(-1e4, 1e4) + noise * torch.randn(z.shape, generator=g)) / T
    logp, ids = torch.log_softmax(t, 1).topk(top, 1)
    ids = ids.int()
    if unused:
        r = torch.rand(ids.shape, generator=g)
        ids[r < 0.1] = -1
        logp[(r > 0.1) & (r < 0.2)] = -math.inf
    return ids, logp


def params(kind, T=1.0, coeff=1.0, floor=FLOOR, flags=0, denominator=0.0):
    d, r = KINDS[kind]
    return B.DistillParams(T, coeff, d, r, floor, flags, denominator)


def run(z, flat, ids, logq, mask, weight, dp, grad=True, in_place=False, loss=None, stats=None, stream=None):
    N, V = z.shape
    dev = flat.cuda()
    before = dev.clone()
    zd = dev[z.storage_offset():].as_strided((N, V), (z.stride(0), 1))
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    wide = torch.full((N, V + 5), 3.0, dtype=z.dtype, device="cuda")
    dz = zd if in_place else wide[:, :V] if grad else None
    kl = torch.full((N + 3,), 9.0, device="cuda")
    loss = torch.full((1,), 99.0, device="cuda") if loss is None else loss
    stats = torch.full((2,), 99, dtype=torch.int64, device="cuda") if stats is None else stats
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.randint(0, 255, (B.workspace_bytes(B.WS_DISTILL, N, V),), dtype=torch.uint8, device="cuda")
    B.mrl_distill_loss_fwd_bwd(zd, cu(ids), cu(logq), cu(mask), cu(weight), dp, dz, kl[:N], loss, stats, status, ws, stream=stream)
    torch.cuda.synchronize()
    assert bool((kl[N:] == 9.0).all())
    if in_place:        # what lies between the rows stays
        inside = torch.zeros(flat.numel(), dtype=torch.bool)
        inside[z.storage_offset():].as_strided((N, V), (z.stride(0), 1)).fill_(True)
        assert torch.equal(dev.cpu()[~inside], before.cpu()[~inside])
    else:
        assert torch.equal(dev.view(torch.uint8), before.view(torch.uint8)) and bool((wide[:, V:] == 3.0).all())
    return {"loss": float(loss), "row_kl": kl[:N].cpu(), "dz": None if dz is None else dz.cpu().clone(), "stats": stats.tolist(),
            "status": int(status)}


def kl_slack(z, ids, logq, T, floor):
    """1 + the largest |ln p - ln q| that a row's terms can have."""
    x = z.double() / T
    ln_p = torch.log_softmax(x, 1)
    used = (ids >= 0) & (logq > -math.inf) & (ids < z.shape[1])
    d = (ln_p.gather(1, ids.long().clamp(0, z.shape[1] - 1)) - logq.double()).abs()
    return 1 + torch.where(used, d, 0.0).nan_to_num(0, 0, 0).amax(1) + abs(math.log(floor)) + math.log(z.shape[1])


def check(z, got, ids, logq, mask, weight, dp, floor=FLOOR):
    V, T = z.shape[1], dp.temperature
    ref = S.distill_loss(z.float(), ids, logq, mask, weight, T, dp.coeff, dp.direction == B.DISTILL_REVERSE, dp.rest == B.REST_EVENT,
                         floor, dp.denominator)
    e = chain(V) + 8 * HALF
    slack = kl_slack(z, ids, logq, T, floor)
    fine = ref["row_kl"].isfinite()
    assert torch.equal(got["row_kl"].isfinite(), fine)
    assert bool(((got["row_kl"].double() - ref["row_kl"]).abs() <= e * slack + HALF * ref["row_kl"].abs())[fine].all())
    assert got["stats"] == [ref["state"].count(1), ref["state"].count(2)]
    if math.isfinite(ref["loss"]):
        w = torch.ones(len(slack)) if weight is None else weight.abs()
        d = dp.denominator if dp.denominator > 0 else max(1, ref["state"].count(1))
        live = torch.tensor([s == 1 for s in ref["state"]])
        tol = abs(dp.coeff) / d * e * float((slack * w)[live].sum()) + 2 * HALF * (abs(ref["loss"]) + ref["size"])
        assert abs(got["loss"] - ref["loss"]) <= tol, (got["loss"], ref["loss"], tol)
    if got["dz"] is not None:
        step = torch.finfo(z.dtype).eps / 2
        slack_g = slack[:, None] if dp.direction == B.DISTILL_REVERSE else 1.0      # the gradient moves with KL_t there
        tol = step * ref["dlogits"].abs() + 4 * e * slack_g * ref["parts"] + 2.0 ** -126
        off = (got["dz"].double() - ref["dlogits"]).abs()
        rows_ok = ref["dlogits"].isfinite().all(1)
        assert bool((off <= tol)[rows_ok].all()), float((off - tol)[rows_ok].max())
        off_rows = torch.tensor([s != 1 for s in ref["state"]])
        assert not bool(got["dz"][off_rows].float().any())
    return ref


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("N,V,dtype,top,T,pad,offset", [
    (1, 1, torch.float32, 1, 1.0, 0, 0), (4, 3, torch.bfloat16, 3, 1.0, 1, 1), (3, 40, torch.float32, 8, 2.0, 0, 1),
    (6, 1003, torch.bfloat16, 20, 0.7, 5, 3), (5, 4096, torch.float32, 128, 1.0, 0, 0), (131, 8000, torch.bfloat16, 20, 1.0, 0, 0),
    (7, 32003, torch.bfloat16, 128, 1.0, 0, 0), (3, 50021, torch.float32, 8, 1.0, 3, 2), (2, 128256, torch.bfloat16, 64, 2.0, 0, 0),
    (2, 151936, torch.float32, 64, 1.0, 0, 0), (330, 5003, torch.bfloat16, 33, 1.0, 3, 1), (320, 4104, torch.float32, 16, 1.0, 8, 0),
    (300, 66000, torch.bfloat16, 64, 1.0, 0, 0), (40, 140000, torch.float32, 5, 1.0, 0, 0),
])
def test_against_the_oracle(kind, N, V, dtype, top, T, pad, offset):
    z, flat = rows(N, V, dtype, N + V, pad, offset)
    T = float(torch.tensor(T))
    ids, logq = lists(z, top, 3, T)
    g = torch.Generator().manual_seed(1)
    mask = (torch.rand(N, generator=g) < 0.8).to(torch.uint8) if N > 3 else None
    weight = torch.rand(N, generator=g) * 2 if N > 2 else None
    if weight is not None:
        weight[0] = 0.0
    dp = params(kind, T, 0.7)
    a = run(z, flat, ids, logq, mask, weight, dp)
    check(z, a, ids, logq, mask, weight, dp)
    assert a["status"] == 0
    b = run(z, flat, ids, logq, mask, weight, dp, in_place=True)
    c = run(z, flat, ids, logq, mask, weight, dp, grad=False)
    assert torch.equal(a["dz"].view(torch.uint8), b["dz"].view(torch.uint8)) and torch.equal(a["row_kl"], b["row_kl"])
    assert a["loss"] == b["loss"] == c["loss"] and torch.equal(a["row_kl"], c["row_kl"]) and a["stats"] == c["stats"]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", sorted(KINDS))
def test_extreme_logits(kind, dtype):
    V, low = 5000, torch.finfo(dtype).min
    z = torch.randn(10, V, generator=torch.Generator().manual_seed(3)).to(dtype)
    ids = torch.arange(8, dtype=torch.int32).expand(10, 8).contiguous()
    logq = torch.log_softmax(torch.randn(10, 9), 1)[:, :8].contiguous()
    z[0, 8:] = -math.inf                # no rest
    z[1, 8:] = low
    z[2] = low                          # uniform
    z[3, :8] = low                      # the listed tokens underflow
    z[4, 0] = 80.0                      # nearly one-hot on a listed token: the rest has e^-80
    z[5, 100] = 80.0                    # and on another
    z[6, 3] = -math.inf                 # a listed token the learner cannot give
    z[7] = -math.inf
    z[8, 5] = math.nan
    z[9, 4000] = math.inf
    dp = params(kind)
    got = run(z, z.view(-1), ids, logq, None, None, dp)
    assert got["row_kl"][7:].isnan().all() and math.isnan(got["loss"]) and got["stats"] == [10, 0]
    assert got["dz"][8:].isnan().any(1).all()
    head = {**got, "row_kl": got["row_kl"][:7], "dz": got["dz"][:7] * 1.0, "loss": math.inf, "stats": [7, 0]}
    dp10 = params(kind, denominator=10.0)
    finite = torch.tensor([0, 1, 2, 4, 5] + ([6] if kind == "reverse" else []))
    pick = lambda t: t[finite]  # noqa: E731
    head = {**head, "row_kl": pick(got["row_kl"]), "dz": pick(got["dz"]), "stats": [len(finite), 0]}
    ref = S.distill_loss(pick(z).float(), pick(ids), pick(logq), None, None, 1.0, 1.0, kind == "reverse", kind != "none", FLOOR, 10.0)
    head["loss"] = ref["loss"]
    check(pick(z), head, pick(ids), pick(logq), None, None, dp10)
    if kind != "reverse":
        assert got["row_kl"][6] == math.inf and got["dz"][6].isfinite().all()
    assert got["dz"][3].isfinite().all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("N", [1, 6, 310])
def test_low_rows_of_several_blocks_in_place(N, kind, dtype):
    V, low = 100003, torch.finfo(dtype).min
    g = torch.Generator().manual_seed(N)
    z = torch.randn(N, V, generator=g).to(dtype)
    z[::2] = low
    z[::2, 99990:] = 0.75 * low       # what the rest of these rows has is far from its first parts
    z[4::6] = -math.inf
    z[4::6, :8] = torch.randn(8, generator=g).to(dtype)
    z[4::6, 50000] = low
    ids = torch.arange(8, dtype=torch.int32).expand(N, 8).contiguous()
    logq = torch.log_softmax(torch.randn(N, 9, generator=g), 1)[:, :8].contiguous()
    dp = params(kind, denominator=5.0)
    a = run(z, z.view(-1), ids, logq, None, None, dp)
    for _ in range(3):
        b = run(z, z.view(-1), ids, logq, None, None, dp, in_place=True)
        assert torch.equal(a["dz"].view(torch.uint8), b["dz"].view(torch.uint8))
        assert torch.equal(a["row_kl"].view(torch.int32), b["row_kl"].view(torch.int32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("V,top,pad,offset", [(33, 8, 0, 0), (1003, 20, 3, 1), (9001, 128, 0, 0), (16000, 33, 0, 0)])
def test_short_rows_of_many(V, top, pad, offset, kind, dtype):
    N, low = 420, torch.finfo(dtype).min
    z, flat = rows(N, V, dtype, V, pad, offset)
    ids, logq = lists(z, top, 4)
    free = torch.ones(N, V, dtype=torch.bool)
    for r in range(0, N, 7):                # rows whose unlisted tokens are masked, one way and the other, some but for a few
        free[r][ids[r][ids[r] >= 0].long()] = False
        free[r, :V // 9 if r % 14 else 0] = False
        z[r][free[r]] = -math.inf if r % 21 else low
    g = torch.Generator().manual_seed(V)
    weight = torch.rand(N, generator=g) + 0.5
    mask = (torch.rand(N, generator=g) < 0.9).to(torch.uint8)
    dp = params(kind, 1.0, 0.7)
    a = run(z, flat, ids, logq, mask, weight, dp)
    check(z, a, ids, logq, mask, weight, dp)
    b = run(z, flat, ids, logq, mask, weight, dp, in_place=True)
    assert torch.equal(a["dz"].view(torch.uint8), b["dz"].view(torch.uint8)) and torch.equal(a["row_kl"], b["row_kl"]) and a["loss"] == b["loss"]


def test_refused_lists_and_empty_rows():
    z, flat = rows(9, 2000, torch.bfloat16, 5)
    ids, logq = lists(z, 70, 1, unused=False)
    ids[1, 69] = 2000
    ids[2, 40] = ids[2, 3]
    logq[3, 5] = math.nan
    logq[4, 5] = math.inf
    ids[5] = -1
    logq[6] = -math.inf
    ids[7, 2], logq[7, 2] = 5000, -math.inf         # an unused place may hold anything
    ids[8, 60], logq[8, 60] = -7, math.nan
    mask = torch.ones(9, dtype=torch.uint8)
    dp = params("forward")
    got = run(z, flat, ids, logq, mask, None, dp)
    assert got["status"] == B.DEV_BAD_TOKEN_ID | B.DEV_BAD_LIST
    ref = check(z, got, ids, logq, mask, None, dp)
    assert ref["state"] == [1, 2, 2, 2, 2, 0, 0, 1, 1]
    mask[1:5] = 0
    got = run(z, flat, ids, logq, mask, None, dp)
    assert got["status"] == 0 and got["stats"] == [3, 0]
    check(z, got, ids, logq, mask, None, dp)
    got = run(z, flat, ids, logq, torch.zeros(9, dtype=torch.uint8), None, dp)
    assert got["loss"] == 0.0 and got["stats"] == [0, 0] and not got["dz"].float().any()


def test_the_same_token_twice_in_every_pair_of_places():
    V, top = 600, 128
    pairs = [(a, b) for a in (0, 1, 31, 32, 63, 64, 95, 96, 127) for b in range(top) if a != b]
    ids = torch.stack([torch.randperm(V)[:top] for _ in pairs]).int()
    for t, (a, b) in enumerate(pairs):
        ids[t, a] = ids[t, b]
    z = torch.randn(len(pairs) + 1, V)
    ids = torch.cat([ids, torch.arange(top, dtype=torch.int32)[None]])
    got = run(z, z.view(-1), ids, torch.full(ids.shape, -5.0), None, None, params("forward"), grad=False)
    assert got["stats"] == [1, len(pairs)] and got["status"] == B.DEV_BAD_LIST


def test_slabs_with_one_denominator_are_the_whole_step():
    z, flat = rows(50, 3001, torch.float32, 2)
    ids, logq = lists(z, 10, 1)
    whole = run(z, flat, ids, logq, None, None, params("reverse"))
    loss, stats = torch.zeros(1, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    parts = []
    for a, b in ((0, 17), (17, 18), (18, 50)):
        p = params("reverse", flags=B.FLAG_ACCUMULATE_LOSS, denominator=float(whole["stats"][0]))
        cut = z[a:b].clone()
        parts.append(run(cut, cut.view(-1), ids[a:b], logq[a:b], None, None, p, loss=loss, stats=stats))
    assert stats.tolist() == whole["stats"]
    assert abs(float(loss) - whole["loss"]) <= 4 * HALF * abs(whole["loss"])
    # Rows of 3,001 floats start on another address in a slab than in the whole, and a row's sum is taken in an order that goes by its address: either is
    # within chain of the exact sum, as `check` has it, so the two are within twice that of one another (and of its rounding, and the slope's).
    e = 2 * (chain(3001) + 8 * HALF) * kl_slack(z, ids, logq, 1.0, FLOOR)
    kl = torch.cat([p["row_kl"] for p in parts])
    assert bool(((kl - whole["row_kl"]).abs() <= e + 2 * HALF * kl.abs()).all())
    ref = S.distill_loss(z.float(), ids, logq, None, None, 1.0, 1.0, True, True, FLOOR, 0.0)
    off = (torch.cat([p["dz"] for p in parts]).double() - whole["dz"].double()).abs()
    assert bool((off <= 4 * e[:, None] * ref["parts"] + 4 * HALF * ref["dlogits"].abs()).all())


def test_slabs_of_aligned_rows_are_the_whole_step_bit_for_bit():
    z, flat = rows(50, 3008, torch.float32, 2)
    ids, logq = lists(z, 10, 1)
    whole = run(z, flat, ids, logq, None, None, params("reverse"))
    parts = []
    for a, b in ((0, 17), (17, 18), (18, 50)):
        cut = z[a:b].clone()
        parts.append(run(cut, cut.view(-1), ids[a:b], logq[a:b], None, None, params("reverse", denominator=float(whole["stats"][0]))))
    assert torch.equal(torch.cat([p["row_kl"] for p in parts]), whole["row_kl"])
    assert torch.equal(torch.cat([p["dz"] for p in parts]), whole["dz"])


def test_no_rows():
    loss, stats = torch.full((1,), 5.0, device="cuda"), torch.full((2,), 5, dtype=torch.int64, device="cuda")
    z, ids, logq = torch.empty(0, 10, device="cuda"), torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, 3, device="cuda")
    B.mrl_distill_loss_fwd_bwd(z, ids, logq, None, None, params("forward", flags=B.FLAG_ACCUMULATE_LOSS), None, None, loss, stats)
    assert float(loss) == 5.0 and stats.tolist() == [5, 5]
    B.mrl_distill_loss_fwd_bwd(z, ids, logq, None, None, params("forward"), None, None, loss, stats)
    assert float(loss) == 0.0 and stats.tolist() == [0, 0]


@pytest.mark.parametrize("kind", sorted(KINDS))
def test_gradient_is_the_slope_of_the_loss(kind):
    """Central differences of the kernel's own loss in float32: h = 2^-4 leaves a third-order term of h^2 / 6 of the row's terms and
    roundings of 2^-24 |loss| / h; a weight and a temperature are on."""
    z, flat = rows(1, 400, torch.float32, 8)
    ids, logq = lists(z, 6, 2, unused=False)
    w, dp = torch.tensor([1.5]), params(kind, 1.25, 0.8)
    base = run(z, flat, ids, logq, None, w, dp)
    h = 2.0 ** -4
    for v in [int(ids[0, 0]), int(ids[0, 5]), int(z.argmin()), 7, 399]:
        up, down = z.clone(), z.clone()
        up[0, v] += h
        down[0, v] -= h
        f = lambda t: run(t, t.reshape(-1), ids, logq, None, w, dp, grad=False)["loss"]  # noqa: E731
        slope = (f(up) - f(down)) / (2 * h)
        size = abs(float(base["dz"][0, v])) + 0.02
        assert abs(slope - float(base["dz"][0, v])) <= h * h * size + 8 * HALF * (abs(base["loss"]) + 1) / h


def test_rows_past_four_gigabytes():
    N, V = 34000, 70000
    z = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    ids = torch.randint(0, V, (N, 1), device="cuda", dtype=torch.int32)
    logq = torch.full((N, 1), math.log(0.5), device="cuda")
    kl, loss = torch.empty(N, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(B.workspace_bytes(B.WS_DISTILL, N, V), dtype=torch.uint8, device="cuda")
    B.mrl_distill_loss_fwd_bwd(z, ids, logq, None, None, params("forward", coeff=float(N)), z, kl, loss, None, None, ws)
    want = 0.5 * math.log(0.5 * V) + 0.5 * math.log(0.5 * V / (V - 1))
    assert float((kl.double() - want).abs().max()) < 32 * chain(V)
    at = z.gather(1, ids.long())
    assert float((at.float() - (1.0 / V - 0.5)).abs().max()) <= 0.5 * 2.0 ** -8
    z.scatter_(1, ids.long(), 0.0)
    rest = 1.0 / V - 0.5 / (V - 1)
    assert abs(float(z.amax()) - rest) <= rest * 2.0 ** -7 and int((z != 0).sum(dtype=torch.int64)) == N * (V - 1)


def test_graph_replay_and_two_streams():
    z, flat = rows(64, 9000, torch.bfloat16, 4)
    ids, logq = (t.cuda() for t in lists(z, 16, 2))
    zd = z.cuda().contiguous()

    def make():
        return dict(dz=torch.zeros_like(zd), kl=torch.zeros(64, device="cuda"), loss=torch.zeros(1, device="cuda"),
                    ws=torch.empty(B.workspace_bytes(B.WS_DISTILL, 64, 9000), dtype=torch.uint8, device="cuda"))

    def call(o, st=None):
        B.mrl_distill_loss_fwd_bwd(zd, ids, logq, None, None, params("reverse"), o["dz"], o["kl"], o["loss"], None, None, o["ws"], stream=st)

    a, b, c = make(), make(), make()
    call(a)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call(b, side)
    for _ in range(3):
        graph.replay()
        call(c, side)
    torch.cuda.synchronize()
    for o in (b, c):
        for k in ("dz", "kl", "loss"):
            assert torch.equal(a[k], o[k]), k
