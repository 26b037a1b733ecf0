"""GPU parity of the gradient norm (mrl_grad_norm) and the AdamW update (mrl_adamw_step) with the float64 oracle.

Tolerances, derived; u = 2^-24.  m: two products, one sum, the gradient's scaling and the rounded constants: 6 u of the
magnitudes of its two parts; v the same with the square: 8 u.  sqrt(v) halves that; the bias corrections, root, sum,
quotient and products of the update: at most 24 u of it with the approximate forms of the root and the quotient (2 units
in the last place each), plus m's error over the denominator.  The parameter adds 3 u of itself, and half a step of its
type where it is rounded.  An 8-bit state is the nearest code (or the code that its dither gives) of a value known to
the same accuracy, or its neighbour where the value is that near the border between two."""
import pytest
import torch

from oracle import step_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
LR, B1, B2, EPS = 1e-3, 0.9, 0.999, 1e-8


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def buf(t, shift, dtype):
    """t on the device, `shift` elements behind the start of an allocation, with guards of NaN (0xff) around it."""
    n = t.numel()
    if dtype in (torch.uint8, E4M3):
        flat = torch.full((n + shift + 64,), 0xFF, dtype=torch.uint8, device="cuda")
        flat[shift:shift + n] = t.view(torch.uint8).cuda()
    else:
        flat = torch.full((n + shift + 64,), float("nan"), dtype=dtype, device="cuda")
        flat[shift:shift + n] = t.to(dtype).cuda()
    return flat, flat[shift:shift + n]


def guards_hold(flat, shift, n):
    outside = torch.cat([flat[:shift], flat[shift + n:]])
    return bool((outside == 0xFF).all()) if flat.dtype == torch.uint8 else bool(torch.isnan(outside).all())


def norm_of(grads, max_norm=1.0, stream=None):
    lst = B.TensorList([B.TensorSlot(grad=g) for g in grads])
    norm, coef = torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")
    ws = torch.full((B.workspace_bytes(B.WS_GRAD_NORM, 0, 0),), 0xFF, dtype=torch.uint8, device="cuda")
    B.mrl_grad_norm(lst, max_norm, norm, coef, ws, stream=stream)
    torch.cuda.synchronize()
    return float(norm), float(coef)


def close_norm(got, grads, max_norm=1.0):
    """float32 runs of at most 64 squares: 66 u of the sum, half that of the root; the float64 rest and two roundings: 2 u."""
    norm, coef = S.grad_norm([g.cpu() for g in grads], max_norm)
    assert abs(got[0] - norm) <= 35 * U * norm and abs(got[1] - coef) <= 35 * U * coef, (got, norm, coef)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("sizes", [[1], [3], [255], [256], [257], [2048], [2049, 1], [16384], [16385, 7, 0, 100000], [3_000_001]])
def test_grad_norm_matches_the_oracle(sizes, dtype):
    for shift in (0, 1):
        grads = [buf(torch.randn(n, generator=torch.Generator().manual_seed(n)), shift, dtype)[1] for n in sizes]
        close_norm(norm_of(grads), grads)
        close_norm(norm_of([g.mul_(1e-3) for g in grads], max_norm=0.5), grads, 0.5)


def test_grad_norm_of_many_tensors_of_both_types():
    g = torch.Generator().manual_seed(1)
    grads = [torch.randn(int(n), generator=g).to(BF16 if k % 3 else F32).cuda()
             for k, n in enumerate(torch.randint(0, 700, (1201,), generator=g))]
    a = norm_of(grads)
    close_norm(a, grads)
    assert norm_of(grads) == a and norm_of(grads, stream=torch.cuda.Stream()) == a
    assert norm_of([]) == (0.0, 1.0) and norm_of(grads, max_norm=0.0)[1] == 1.0 and norm_of(grads, max_norm=-1.0)[1] == 1.0


def test_grad_norm_range_and_non_finite_values():
    for dtype in (BF16, F32):
        for size in (1e-30, 1e-22, 1e18, 1e25, 3e38):          # squares that leave float32 on either side
            grads = [torch.full((1000,), size).to(dtype).cuda(), torch.zeros(513, dtype=dtype, device="cuda")]
            norm, _ = S.grad_norm([g.cpu() for g in grads], 1.0)
            got = norm_of(grads)
            assert abs(got[0] - norm) <= 35 * U * norm if norm < 3.4e38 else got[0] == float("inf")
        for bad in (float("inf"), float("nan")):
            grads = [torch.ones(5000, dtype=dtype, device="cuda"), torch.ones(77, dtype=dtype, device="cuda")]
            grads[1][76] = bad
            norm, coef = norm_of(grads)
            assert not norm < float("inf") and coef != coef
    grads = [torch.zeros(100, device="cuda")]
    assert norm_of(grads) == (0.0, 1.0) and norm_of(grads, max_norm=float("inf")) == (0.0, 1.0)
    assert norm_of([torch.full((100,), 2.0, device="cuda")], max_norm=float("inf")) == (20.0, 1.0)


class Case:
    """One tensor with its state, in guarded buffers, and a float64 copy of where it starts."""

    def __init__(self, n, param, master, grad, state, seed, shift=0, decay=0.01, rng_first=0, size=1e-2):
        g = torch.Generator().manual_seed(seed)
        r = lambda: torch.randn(n, generator=g)  # noqa: E731
        self.n, self.state, self.decay, self.rng_first, self.shift, self.ptype = n, state, decay, rng_first, shift, param
        self.b = {"grad": buf(r() * size, shift, grad)}
        first = r() * 0.5
        self.b["param"] = buf(first, shift, param)
        if master:
            self.b["master"] = buf(first, shift, F32)
        m, v = r() * size * 0.3, (r() * size) ** 2
        if n > 3:
            v[1], m[2] = 0.0, 0.0
            if n > 600:
                m[256:512], v[256:512] = 0.0, 0.0             # a whole block without a past
                self.b["grad"][1][256:300] = 0.0
        if state == E4M3:
            for name, s in (("m", m), ("v", v.sqrt())):
                scale, each = S.block_scales(s.double())
                self.b[name] = buf((s.double() / each).float().to(E4M3), shift, E4M3)
                self.b[name + "_scale"] = buf(scale.float(), shift, F32)
        else:
            self.b["m"], self.b["v"] = buf(m, shift, F32), buf(v, shift, F32)
        self.start = {k: t[1].clone() for k, t in self.b.items()}
        self.slot = B.TensorSlot(**{k: t[1] for k, t in self.b.items()}, weight_decay=decay, rng_first=rng_first)

    def state64(self, name):
        t = self.start[name]
        if self.state != E4M3:
            return t.cpu().double()
        s = t.view(E4M3).cpu().double() * self.start[name + "_scale"].cpu().double().repeat_interleave(S.STATE_BLOCK)[:self.n]
        return s if name == "m" else s * s

    def check(self, step, scale=1.0, seeded=None, lr=LR):
        got = {k: t[1].cpu() for k, t in self.b.items()}
        for k, (flat, _) in self.b.items():
            assert guards_hold(flat, self.shift, got[k].numel()), k
        assert torch.equal(got["grad"], self.start["grad"].cpu())
        master = "master" in self.b
        p0 = self.start["master" if master else "param"].cpu().double()
        m0, v0, g = self.state64("m"), self.state64("v"), self.start["grad"].cpu().double() * scale
        decay = float(torch.tensor(self.decay, dtype=F32))
        p, m, v, up = S.adamw(p0, g, m0, v0, lr, B1, B2, EPS, decay, step)
        em = 6 * U * (B1 * m0.abs() + (1 - B1) * g.abs()) + 1e-44
        ev = 8 * U * v + 1e-44
        den = torch.sqrt(v / (1 - B2 ** step)) + EPS
        ep = 3 * U * p.abs() + lr * (24 * U * up.abs() + em / (1 - B1 ** step) / den + 4 * U * decay * p0.abs())
        rm, rv, rp = S.dithers(self.n, seeded, step, self.rng_first) if seeded is not None else (None, None, None)
        full = got["master"] if master else got["param"]
        if full.dtype == F32:
            assert bool(((full.double() - p).abs() <= ep).all()), "param"
        if master:
            assert torch.equal(got["param"], got["master"].to(BF16))
        elif full.dtype == BF16:
            grid = S.bf16_grid(p.abs())
            to, border = S.grid_target(p.abs(), grid, rp)
            sure = border > ep / grid + 1e-9
            assert torch.equal(full.double()[sure], (to * torch.sign(p))[sure]), "bf16 param"
            assert bool(((full.double() - p).abs() <= grid * (1 if seeded is not None else 0.5) + ep + 1e-40).all())
        if self.state == F32:
            assert bool(((got["m"].double() - m).abs() <= em).all()) and bool(((got["v"].double() - v).abs() <= ev).all())
            return
        # (each term of v is off by up to 2^-149 where it leaves float32's normal range, 1e-44 in all, and
        # |sqrt(a) - sqrt(b)| <= sqrt(|a - b|): a root is off by up to 1e-22 there)
        for name, s, e, dither in (("m", m, em, rm), ("v", torch.sqrt(v), torch.sqrt(v) * 5 * U + 1e-22, rv)):
            scale64, each = S.block_scales(s)
            e_top = torch.stack([b.max() for b in e.split(S.STATE_BLOCK)])
            assert bool(((got[name + "_scale"].double() - scale64).abs() <= 3 * U * scale64 + e_top / 448).all()), name
            pos = s / each
            rel = 6 * U + (e_top / (scale64 * 448)).repeat_interleave(S.STATE_BLOCK)[:self.n]
            ep_pos = pos.abs() * rel + e / each
            grid = S.e4m3_grid(pos.abs())
            to, border = S.grid_target(pos.abs(), grid, dither, top=448.0)
            if name == "v":
                to = torch.where((pos > 0) & (to == 0), torch.tensor(2.0 ** -9, dtype=torch.float64), to)
            code = got[name].view(E4M3).double()
            # (the dither's grid moves values below 2^-6 by 2^-6 in float32: 2^-30 against codes 2^-9 apart)
            sure = border > ep_pos / grid + 2.0 ** -20
            assert torch.equal(code[sure], (to * torch.sign(pos))[sure]), name
            far = grid * (1.0 if dither is not None else 0.5) + 2 * ep_pos + 1e-9
            if name == "v":
                far = far.clamp_min(2.0 ** -9)
            assert bool(((code - pos).abs() <= far).all()), name


KINDS = [(p, mst, g, s) for p, mst in ((F32, False), (BF16, False), (BF16, True)) for g in (F32, BF16) for s in (F32, E4M3)]


def step_of(cases, step=3, seeded=None, scale=None, lr=LR, stream=None, **kw):
    ap = B.AdamwParams(lr=lr, beta1=B1, beta2=B2, eps=EPS, step=step, seed=seeded or 0,
                       rounding=B.ROUND_NEAREST if seeded is None else B.ROUND_SEEDED)
    for k, t in kw.items():
        setattr(ap, k, t)
    gs = None if scale is None else torch.tensor([scale], dtype=F32).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.full((B.workspace_bytes(B.WS_ADAMW, 0, 0),), 0xFF, dtype=torch.uint8, device="cuda")
    B.mrl_adamw_step(B.TensorList([c.slot for c in cases]), ap, gs, status, ws, stream=stream)
    torch.cuda.synchronize()
    return int(status)


@pytest.mark.parametrize("param,master,grad,state", KINDS)
@pytest.mark.parametrize("seeded", [None, 12345])
def test_adamw_matches_the_oracle(param, master, grad, state, seeded):
    for shift in (0, 1, 8):
        sizes = [1, 2, 7, 8, 255, 256, 257, 1000, 2048, 5003]
        cases = [Case(n, param, master, grad, state, seed=n, shift=shift, rng_first=1000 * k, decay=0.0 if k % 3 else 0.1)
                 for k, n in enumerate(sizes)]
        assert step_of(cases, seeded=seeded, scale=0.5) == 0
        for c in cases:
            c.check(3, 0.5, seeded)


def test_many_tensors_of_all_kinds_in_one_call():
    g = torch.Generator().manual_seed(4)
    sizes = torch.randint(0, 900, (1000,), generator=g).tolist()
    cases = [Case(n, *KINDS[k % len(KINDS)], seed=k, shift=k % 2, rng_first=500 * k) for k, n in enumerate(sizes)]
    step_of(cases, step=1, seeded=9)
    for c in cases[::7] + cases[-30:]:
        if c.n:
            c.check(1, 1.0, 9)
    big = Case(1_000_003, BF16, False, BF16, F32, seed=5)
    step_of([big], step=1000)
    big.check(1000)


def test_first_step_from_empty_states():
    for state in (F32, E4M3):
        c = Case(700, F32, False, F32, state, seed=3)
        for k in ("m", "v", "m_scale", "v_scale"):
            if k in c.b:
                c.b[k][1].zero_()
                c.start[k].zero_()
        step_of([c], step=1)
        c.check(1)


def test_gradients_that_are_tiny_or_zero():
    for size in (0.0, 1e-30, 1e-12):
        for kind in KINDS:
            c = Case(520, *kind, seed=6, size=size)
            step_of([c], step=2, seeded=7)
            c.check(2, 1.0, 7)


@pytest.mark.parametrize("scale", [float("nan"), float("inf")])
def test_a_scale_that_is_not_finite_skips_the_step(scale):
    cases = [Case(300, *kind, seed=2) for kind in KINDS]
    count = torch.tensor([4], dtype=torch.int64, device="cuda")
    assert step_of(cases, scale=scale) == B.DEV_NONFINITE_GRAD
    assert step_of(cases, scale=scale, step_dev=count.data_ptr()) == B.DEV_NONFINITE_GRAD
    assert int(count) == 4
    for c in cases:
        for k, t in c.b.items():
            assert torch.equal(t[1].view(torch.uint8), c.start[k].view(torch.uint8)), k


def test_step_and_learning_rate_on_the_device():
    for seeded in (None, 77):
        for kind in KINDS:
            c = Case(600, *kind, seed=8)
            count, lr = torch.tensor([6], dtype=torch.int64, device="cuda"), torch.tensor([2e-3], device="cuda")
            step_of([c], step=0, seeded=seeded, step_dev=count.data_ptr(), lr_dev=lr.data_ptr())
            assert int(count) == 7
            c.check(7, 1.0, seeded, lr=float(lr))
    count = torch.tensor([6], dtype=torch.int64, device="cuda")
    step_of([], step_dev=count.data_ptr())
    assert int(count) == 7


def test_replayed_steps_are_the_steps_of_direct_calls():
    """Clip factor and update in one graph, counter and gradients on the device: three replays against three direct calls."""
    kinds = [(BF16, False, BF16, E4M3), (BF16, True, BF16, F32), (F32, False, F32, E4M3)]
    a, b = ([Case(n, *k, seed=n, rng_first=n) for n, k in zip((3000, 1111, 700), kinds)] for _ in range(2))
    grads = [[torch.randn(c.n, generator=torch.Generator().manual_seed(50 + t)).to(c.b["grad"][1].dtype).cuda() for c in a]
             for t in range(3)]
    lists = [B.TensorList([c.slot for c in cs]) for cs in (a, b)]
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    coef, ws = torch.zeros(1, device="cuda"), torch.empty(B.workspace_bytes(B.WS_GRAD_NORM, 0, 0), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(B.workspace_bytes(B.WS_ADAMW, 0, 0), dtype=torch.uint8, device="cuda")
    params = lambda **kw: B.AdamwParams(lr=LR, beta1=B1, beta2=B2, eps=EPS, seed=5, rounding=B.ROUND_SEEDED, **kw)  # noqa: E731
    live = params(step_dev=count.data_ptr())

    def step(stream=None):
        B.mrl_grad_norm(lists[1], 1.0, None, coef, ws, stream=stream)
        B.mrl_adamw_step(lists[1], live, coef, None, ws2, stream=stream)

    side = torch.cuda.Stream()
    step(side)
    side.synchronize()
    count.zero_()
    for c in b:                                   # back to the start: the warm-up was a step
        for k, t in c.b.items():
            t[1].copy_(c.start[k])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for t in range(3):
        for cs in (a, b):
            for c, g in zip(cs, grads[t]):
                c.b["grad"][1].copy_(g)
        B.mrl_grad_norm(lists[0], 1.0, None, coef, ws)
        B.mrl_adamw_step(lists[0], params(step=t + 1), coef)
        graph.replay()
        torch.cuda.synchronize()
        assert int(count) == t + 1
    for x, y in zip(a, b):
        for k in x.b:
            assert torch.equal(x.b[k][1].view(torch.uint8), y.b[k][1].view(torch.uint8)), k


def test_seeded_rounding_keeps_small_updates_in_the_mean():
    """lr 1e-6 on bf16 weights near 0.5 (2^-9 apart below, 2^-8 above): every update is below half a step.  The mean of n
    seeded roundings is the exact mean within 5 standard deviations, step / (2 sqrt(n)) each."""
    n = 200_000
    c = Case(n, BF16, False, F32, F32, seed=1, decay=0.0)
    c.b["param"][1].fill_(0.375)
    c.b["grad"][1].fill_(1.0)
    c.b["m"][1].zero_(), c.b["v"][1].zero_()
    step_of([c], step=1, seeded=3, lr=1e-5)
    p = c.b["param"][1].double()
    grid = 2.0 ** -9
    assert sorted(p.unique().tolist()) == [0.375 - grid, 0.375]
    assert abs(float(p.mean()) - (0.375 - 1e-5)) <= 5 * grid * (1e-5 / grid) ** 0.5 / n ** 0.5 + 2 * U
    c.b["param"][1].fill_(0.375)
    step_of([c], step=1, lr=1e-5)
    assert bool((c.b["param"][1] == 0.375).all())


def _float32_step(state, grad, scale, step, seeded):
    """The moments and their codes by torch's float32 operations, one after the other as the formula stands."""
    block = lambda t: t.view(-1, B.STATE_BLOCK)  # noqa: E731
    g = grad.float() * scale
    m = (block(state["m"].view(E4M3).float()) * state["m_scale"][:, None]).view(-1)
    v = (block(state["v"].view(E4M3).float()) * state["v_scale"][:, None]).view(-1)
    v = v * v
    m, v = B1 * m + (1.0 - B1) * g, B2 * v + (1.0 - B2) * (g * g)
    out = {}
    dither = S.dithers(64, seeded, step, 0) if seeded is not None else None      # (checked below for what it covers)
    for k, (name, s) in enumerate((("m", m), ("v", v.sqrt()))):
        sc = (block(s.abs()).amax(1) * torch.tensor(1.0 / 448.0, dtype=F32, device="cuda")).clamp_min(2.0 ** -126)
        y = (block(s) * (1.0 / sc)[:, None]).view(-1)
        if dither is None:
            q = y.clamp(-448, 448).to(E4M3)
        else:
            y = y[:64]
            a = y.abs()
            up = torch.where(a < 2.0 ** -6, 2.0 ** -6, 0.0).float()
            z = (((a + up).view(torch.int32) + (dither[k].int().cuda() << 4)) & ~0xFFFFF).view(F32) - up
            q = torch.copysign(z.clamp(max=448.0), y).to(E4M3)
        if name == "v":
            q = torch.where((y > 0) & (q.float() == 0), 2.0 ** -9, q.float()).to(E4M3)
        out[name], out[name + "_scale"] = q, sc
    return out


@pytest.mark.parametrize("seeded", [None, 31])
def test_codes_are_those_of_the_float32_operations_bit_for_bit(seeded):
    """A million elements over three steps: scales and codes equal those of single float32 operations in the formula's order
    (with seeded rounding the first 64 codes, whose dithers are formed here one by one)."""
    c = Case(1 << 20, F32, False, BF16, E4M3, seed=11)
    for step in (4, 5, 6):
        state = {k: c.b[k][1].clone() for k in ("m", "v", "m_scale", "v_scale")}
        grad = torch.randn(c.n, generator=torch.Generator(device="cuda").manual_seed(step), device="cuda") * 10.0 ** -step
        c.b["grad"][1].copy_(grad)
        want = _float32_step(state, c.b["grad"][1], torch.tensor([0.37], device="cuda"), step, seeded)
        step_of([c], step=step, seeded=seeded, scale=0.37)
        for k in ("m", "v", "m_scale", "v_scale"):
            n = want[k].numel()
            assert torch.equal(c.b[k][1][:n].view(torch.uint8), want[k].view(torch.uint8)), (k, step)


@pytest.mark.parametrize("param,master,grad,state", KINDS)
@pytest.mark.parametrize("tail", [0, 77])
def test_large_calls_give_what_their_pieces_give_alone(param, master, grad, state, tail):
    """A call of more than 9.7 M elements gives its CTAs longer runs: bit for bit the results of calls of fewer."""
    n, cut = 256 * 40_000 + tail, 256 * 13_001
    g = torch.Generator(device="cuda").manual_seed(5)
    start = {"grad": torch.randn(n, generator=g, device="cuda").to(grad), "param": torch.randn(n, generator=g, device="cuda").to(param)}
    if master:
        start["master"] = start["param"].float()
    if state == E4M3:
        for name in ("m", "v"):
            start[name] = torch.randint(0, 0x7F, (n,), generator=g, device="cuda", dtype=torch.uint8).view(E4M3)
            start[name + "_scale"] = torch.rand(-(-n // 256), generator=g, device="cuda") * 1e-4
    else:
        start["m"], start["v"] = torch.randn(n, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    large, parts = ({k: t.clone() for k, t in start.items()} for _ in range(2))

    def slot(tensors, lo, hi):
        of = {k: t[lo // 256:-(-hi // 256)] if k.endswith("_scale") else t[lo:hi] for k, t in tensors.items()}
        return B.TensorSlot(**of, weight_decay=0.01, rng_first=100 + lo // 2)

    ap = B.AdamwParams(lr=LR, beta1=B1, beta2=B2, eps=EPS, step=3, seed=9, rounding=B.ROUND_SEEDED)
    B.mrl_adamw_step(B.TensorList([slot(large, 0, n)]), ap)
    for lo in range(0, n, cut):
        B.mrl_adamw_step(B.TensorList([slot(parts, lo, min(n, lo + cut))]), ap)
    torch.cuda.synchronize()
    for k in start:
        assert torch.equal(large[k].view(torch.uint8), parts[k].view(torch.uint8)), k
        assert k == "grad" or not torch.equal(large[k].view(torch.uint8), start[k].view(torch.uint8)), k


def test_a_state_that_is_not_finite_stays_in_its_block():
    for kind in KINDS:
        for seeded in (None, 3):
            c, d = (Case(1024, *kind, seed=12) for _ in range(2))
            c.b["grad"][1][300] = float("nan")
            c.b["grad"][1][700] = float("inf")
            for one in (c, d):
                step_of([one], seeded=seeded)
            name = "master" if "master" in c.b else "param"
            p, q = c.b[name][1], d.b[name][1]
            assert bool(torch.isnan(p[300])) and bool(torch.isnan(p[700]))        # inf / inf
            rest = torch.ones(1024, dtype=torch.bool, device="cuda")
            rest[[300, 700]] = False
            assert torch.equal(p[rest], q[rest])
            for k in ("m", "v"):
                a, b = c.b[k][1], d.b[k][1]
                assert torch.equal(a[:256], b[:256]) and torch.equal(a[768:], b[768:])
                if kind[3] == E4M3:
                    assert int(a.view(torch.uint8)[300]) & 0x7F == 0x7F
