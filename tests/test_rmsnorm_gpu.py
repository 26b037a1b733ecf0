"""GPU parity of the norm in front of the LM head (mrl_rmsnorm_residual_fwd / _bwd) with the float64 oracle.

Tolerances, derived.  u = 2^-24 is half a float32 step relative to the value.  A row's sum of squares is a sum of
non-negative float32 terms: its relative error is at most (longest chain of additions) u; the longest chain of any
kernel is 16 additions in a thread, 5 shuffles and 32 warps, or H / 512 columns in the looping kernel.  The square root
halves it; the float reciprocal of H, the addition of eps, rsqrtf (2 units in the last place = 4 u), and the products
and the sum that make h and y add at most 10 u.  So y before its rounding is off by at most (chain / 2 + 10) u of itself, and
rounding to the row's type adds half a step, eps / 2 of the value."""
import pytest
import torch

from oracle import step_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def chain(H):
    return max(53, H / 512 + 60)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2 if dtype != F32 else U


def rows(N, H, dtype, seed, pad=0, shift=0, scale=1.0):
    """[N, H] rows, H + pad apart, the first `shift` elements behind the start of an allocation."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.full((N * (H + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    t = flat[shift:shift + N * (H + pad)].view(N, H + pad)[:, :H]
    t.copy_((torch.randn(N, H, generator=g) * scale).to(dtype))
    return t


def within(got, want, tol, name):
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{name}: {int(bad.sum())} values, worst {float((err / tol.clamp_min(1e-300))[bad].max())} x tolerance"


def check_codes(q, scales, y, group, rel, name="y8"):
    """Codes against the unrounded y of the oracle: the nearest value, or its neighbour where y is that near a border."""
    want_s, each = S.group_scales(y, group)
    within(scales, want_s, want_s * rel, "scales")
    got = q.view(torch.float8_e4m3fn).cpu().double()
    pos = y / each
    step = S.e4m3_grid(pos.abs())
    to, border = S.grid_target(pos.abs(), step, top=448.0)
    sure = border > pos.abs() / step * rel + 1e-9
    assert torch.equal(got[sure], (to * torch.sign(pos))[sure]), name
    assert bool(((got - pos).abs() <= step * (0.5 + 16 * rel)).all()), name


def run_fwd(x, res, w, offset=0.0, eps=1e-6, group=0, want=("h", "y", "rstd"), pad=0, shift=0, stream=None, place=None):
    N, H = x.shape
    np = B.NormParams(eps, offset, group, 0)
    out = dict(place or {})
    for k in ("h", "y"):
        if k in want and k not in out:
            out[k] = rows(N, H, x.dtype, 9, pad, shift)
    if "q" in want:
        wide = torch.full((N * (H + pad) + shift,), 0x55, dtype=torch.uint8, device="cuda")
        out["q"] = wide[shift:].view(N, H + pad)[:, :H]
        out["q_wide"] = wide
        out["scales"] = torch.full((N, -(-H // group) if group else 1), float("nan"), device="cuda")
    if "rstd" in want:
        out["rstd"] = torch.full((N,), float("nan"), device="cuda")
    B.mrl_rmsnorm_residual_fwd(x, res, w, np, out.get("h"), out.get("y"), out.get("q"), out.get("scales"), out.get("rstd"),
                               stream=stream)
    torch.cuda.synchronize()
    return out


def check_fwd(x, res, w, out, ref, offset, group):
    H = x.shape[1]
    h, rstd, y = ref
    rel = (chain(H) / 2 + 10) * U
    tiny = 1e-37
    if "rstd" in out:
        within(out["rstd"], rstd, rstd * rel, "rstd")
    if "h" in out:
        within(out["h"], h, h.abs() * (half_step(x.dtype) + U) + tiny, "h")
    if "y" in out:
        within(out["y"], y, y.abs() * (half_step(x.dtype) * (1 + 1e-3) + rel) + tiny, "y")
    if "q" in out:
        check_codes(out["q"], out["scales"], y, group, 2 * rel + 4 * U)


WIDTHS = [1, 2, 3, 31, 33, 64, 100, 127, 128, 257, 512, 1000, 1024, 1027, 2501, 4096, 5128, 8192, 16384]


@pytest.mark.parametrize("H", WIDTHS)
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
def test_forward_matches_the_oracle_over_widths(H, dtype, wdtype):
    for N, residual, offset, group in ((1, False, 0.0, 0), (5, True, 1.0, 32), (67, True, 0.0, 128), (3, False, 1.0, 256), (2, True, 0.0, 64)):
        x, res = rows(N, H, dtype, H + N), rows(N, H, dtype, H + N + 1, scale=3.0) if residual else None
        w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(wdtype).cuda()
        ref = S.rmsnorm_residual_fwd(x, res, w, offset, float(torch.tensor(1e-6, dtype=F32)))
        want = ("h", "y", "rstd", "q") if N != 67 else ("h", "q")
        check_fwd(x, res, w, run_fwd(x, res, w, offset, group=group, want=want), ref, offset, group)


@pytest.mark.parametrize("H", [16385, 16392, 20000, 40001])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_forward_of_very_wide_rows(H, dtype):
    for N, group in ((3, 0), (2, 256)):
        x, res = rows(N, H, dtype, 1), rows(N, H, dtype, 2)
        w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
        ref = S.rmsnorm_residual_fwd(x, res, w, 0.0, float(torch.tensor(1e-6, dtype=F32)))
        check_fwd(x, res, w, run_fwd(x, res, w, group=group, want=("h", "y", "rstd", "q")), ref, 0.0, group)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (5, 3), (8, 0), (8, 8), (64, 4), (16, 16)])
def test_row_strides_and_addresses(dtype, pad, shift):
    for N, H in ((6, 256), (4, 1024), (3, 999)):
        x, res = rows(N, H, dtype, 3, pad, shift), rows(N, H, dtype, 4, pad, shift)
        w_at = torch.empty(H + shift, dtype=dtype, device="cuda")
        w_at[shift:] = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
        w = w_at[shift:]
        ref = S.rmsnorm_residual_fwd(x, res, w, 0.0, float(torch.tensor(1e-6, dtype=F32)))
        out = run_fwd(x, res, w, group=128, want=("h", "y", "rstd", "q"), pad=pad, shift=shift)
        check_fwd(x, res, w, out, ref, 0.0, 128)
        for t in (out["h"], out["y"]):          # what lies between the rows stays as it was
            wide = t.as_strided((N, H + pad), (H + pad, 1))
            assert bool(torch.isnan(wide[:, H:].float()).all())
        between = out["q"].as_strided((N - 1, H + pad), (H + pad, 1))[:, H:]
        assert bool((between == 0x55).all())


@pytest.mark.parametrize("H", [1, 2, 3, 5, 7, 8, 9, 17])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_less_than_a_granule_at_any_address(H, dtype):
    w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
    for shift in range(9):
        for pad in (0, 1, 3):
            x, res = rows(21, H, dtype, 3, pad, shift), rows(21, H, dtype, 4, pad, shift)
            ref = S.rmsnorm_residual_fwd(x, res, w, 0.0, float(torch.tensor(1e-6, dtype=F32)))
            out = run_fwd(x, res, w, group=32, want=("h", "y", "rstd", "q"), pad=pad, shift=shift)
            check_fwd(x, res, w, out, ref, 0.0, 32)
            back = run_bwd(res, None, x, w, out["rstd"], dx=rows(21, H, dtype, 5, pad, shift))
            check_bwd(res, None, x, w, out["rstd"], back)
            for t in (out["h"], out["y"], back["dx"]):
                assert bool(torch.isnan(t.as_strided((21, H + pad), (H + pad, 1))[:, H:].float()).all())


@pytest.mark.parametrize("H", [256, 1001, 4096, 16400])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_outputs_over_inputs(H, dtype):
    N = 33
    w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
    apart = run_fwd(rows(N, H, dtype, 1), rows(N, H, dtype, 2), w, want=("h", "y", "rstd", "q"), group=128)
    for swap in (False, True):
        x, res = rows(N, H, dtype, 1), rows(N, H, dtype, 2)
        out = run_fwd(x, res, w, want=("rstd", "q"), group=128, place={"h": x, "y": res} if swap else {"h": res, "y": x})
        for k in ("h", "y", "rstd", "q", "scales"):
            assert torch.equal(out[k], apart[k]), k
    dy, dh, h = (rows(N, H, dtype, s) for s in (3, 4, 5))
    rstd = apart["rstd"]
    want = run_bwd(dy, dh, h, w, rstd)
    for at in range(3):
        ins = [t.clone() for t in (dy, dh, h)]
        got = run_bwd(*ins, w, rstd, dx=ins[at])
        assert torch.equal(got["dx"], want["dx"]) and torch.equal(got["dw"], want["dw"])


def test_no_rows_and_one_row():
    x = torch.empty(0, 64, dtype=BF16, device="cuda")
    w = torch.ones(64, device="cuda")
    np = B.NormParams(1e-6, 0.0, 0, 0)
    B.mrl_rmsnorm_residual_fwd(x, None, w, np, y=torch.empty_like(x), rstd=torch.empty(0, device="cuda"))
    dw = torch.full((64,), 5.0, device="cuda")
    acc = B.NormParams(1e-6, 0.0, 0, B.FLAG_ACCUMULATE_DW)
    B.mrl_rmsnorm_residual_bwd(x, None, x, w, torch.empty(0, device="cuda"), acc, torch.empty_like(x), dw)
    assert bool((dw == 5.0).all())
    B.mrl_rmsnorm_residual_bwd(x, None, x, w, torch.empty(0, device="cuda"), np, torch.empty_like(x), dw)
    assert bool((dw == 0.0).all())


@pytest.mark.parametrize("H", [33, 1024, 4096, 16401])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_of_zeros_huge_tiny_and_non_finite_values(H, dtype):
    x = rows(8, H, dtype, 1)
    x[1] = 0.0
    x[2] *= 1e25                    # the squares leave float32, the row does not
    x[3] *= 1e-25                   # eps decides
    x[4, H // 2] = float("inf")
    x[5, H - 1] = float("nan")
    x[6] = -3e38 if dtype == F32 else -3.3e38
    w = (1.0 + 0.1 * torch.randn(H, generator=torch.Generator().manual_seed(7))).to(dtype).cuda()
    ref = S.rmsnorm_residual_fwd(x, None, w, 0.0, float(torch.tensor(1e-6, dtype=F32)))
    out = run_fwd(x, None, w, want=("y", "rstd", "q"), group=0)
    rel = (chain(H) / 2 + 10) * U
    for t in (0, 1, 2, 3, 6, 7):
        # (a float32 reciprocal root of 3e38 lies below the normal range: 2^-149 of absolute rounding there)
        within(out["rstd"][t:t + 1], ref[1][t:t + 1], ref[1][t:t + 1] * rel + 2.0 ** -149, f"rstd of row {t}")
        slack = ref[0][t].abs() * 2.0 ** -149 * 2
        within(out["y"][t], ref[2][t], ref[2][t].abs() * (half_step(dtype) * (1 + 1e-3) + rel) + slack + 1e-37, f"y of row {t}")
    check_codes(out["q"][[0, 1, 2, 3, 7]], out["scales"][[0, 1, 2, 3, 7]], ref[2][[0, 1, 2, 3, 7]], 0, 2 * rel + 4 * U)
    y4, y5 = out["y"][4].float().cpu(), out["y"][5].float().cpu()
    assert bool(torch.isnan(y4[H // 2])) and bool((y4[torch.arange(H) != H // 2] == 0).all())     # inf / inf; finite / inf
    assert bool(torch.isnan(y5).all())
    assert int(out["q"][4, H // 2]) & 0x7F == 0x7F and bool((out["q"][5] & 0x7F == 0x7F).all())
    assert int((out["q"][4] & 0x7F != 0).sum()) == 1


def run_bwd(dy, dh, h, w, rstd, offset=0.0, flags=0, dx=None, dw=None, want_dw=True, stream=None):
    N, H = dy.shape
    np = B.NormParams(1e-6, offset, 0, flags)
    dx = torch.full((N, H), float("nan"), dtype=dy.dtype, device="cuda") if dx is None else dx
    dw = torch.full((H,), float("nan"), device="cuda") if dw is None and want_dw else dw
    ws = torch.full((B.workspace_bytes(B.WS_RMSNORM_BWD, N, 0, H),), 0xFF, dtype=torch.uint8, device="cuda") if want_dw else None
    B.mrl_rmsnorm_residual_bwd(dy, dh, h, w, rstd, np, dx, dw, ws, stream=stream)
    torch.cuda.synchronize()
    return {"dx": dx, "dw": dw}


def check_bwd(dy, dh, h, w, rstd, out, offset=0.0, dw0=None):
    """dx: 12 u of the sum of its parts' magnitudes, the inner mean's chain of additions on its part, the type's half step.
    dweight: a chain of N / 148 rows in a CTA, at most 2,400 partials in 8 lanes, and the 8 lanes, u each of the sum of magnitudes."""
    N, H = dy.shape
    dx, ddw, parts, mags = S.rmsnorm_residual_bwd(dy, dh, h, w, offset, rstd)
    within(out["dx"], dx, parts * (chain(H) + 12) * U + dx.abs() * half_step(dy.dtype) * (1 + 1e-3) + 1e-37, "dx")
    if out["dw"] is not None:
        start = torch.zeros(H, dtype=torch.float64) if dw0 is None else dw0.double().cpu()
        within(out["dw"], ddw + start, (mags * (N / 148 + 320) + start.abs() * 2) * U + 1e-37, "dweight")


@pytest.mark.parametrize("H", WIDTHS + [16385, 20000])
@pytest.mark.parametrize("dtype,wdtype", [(BF16, BF16), (F32, F32), (BF16, F32)])
def test_backward_matches_the_oracle_over_widths(H, dtype, wdtype):
    for N, through, offset in ((1, False, 0.0), (7, True, 1.0), (700, True, 0.0)):
        if N * H > 4_000_000:
            N = 40
        dy, h = rows(N, H, dtype, 1), rows(N, H, dtype, 2, scale=2.0)
        dh = rows(N, H, dtype, 3) if through else None
        w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(wdtype).cuda()
        rstd = S.rmsnorm_residual_fwd(h, None, w, offset, 1e-6)[1].float().cuda()
        out = run_bwd(dy, dh, h, w, rstd, offset)
        check_bwd(dy, dh, h, w, rstd, out, offset)
        alone = run_bwd(dy, dh, h, w, rstd, offset, want_dw=False)
        assert torch.equal(alone["dx"], out["dx"])
        again = run_bwd(dy, dh, h, w, rstd, offset)
        assert torch.equal(again["dx"], out["dx"]) and torch.equal(again["dw"], out["dw"])      # bit for bit
        start = torch.randn(H, generator=torch.Generator().manual_seed(8)).cuda()
        acc = run_bwd(dy, dh, h, w, rstd, offset, flags=B.FLAG_ACCUMULATE_DW, dw=start.clone())
        check_bwd(dy, dh, h, w, rstd, acc, offset, dw0=start)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad,shift", [(0, 1), (5, 3), (8, 0), (8, 8), (16, 16)])
def test_backward_row_strides_and_addresses(dtype, pad, shift):
    for N, H in ((6, 256), (400, 1024), (3, 999)):
        dy, dh, h = (rows(N, H, dtype, s, pad, shift) for s in (1, 2, 3))
        w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
        rstd = S.rmsnorm_residual_fwd(h, None, w, 0.0, 1e-6)[1].float().cuda()
        dx = rows(N, H, dtype, 4, pad, shift)
        out = run_bwd(dy, dh, h, w, rstd, dx=dx)
        check_bwd(dy, dh, h, w, rstd, out)
        assert bool(torch.isnan(dx.as_strided((N, H + pad), (H + pad, 1))[:, H:].float()).all())


MANY = [(20000, 64), (9000, 320), (7000, 512), (3000, 1000), (3000, 1024), (2500, 1027), (2100, 4096), (2100, 4095), (700, 8192),
        (450, 16384)]


def random_rows(N, H, dtype, seed, pad=0, scale=1.0):
    """As rows(), made on the device (the oracle reads back what it needs)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = torch.full((N, H + pad), float("nan"), dtype=dtype, device="cuda")
    wide[:, :H] = torch.randn(N, H, generator=g, device="cuda") * scale
    return wide[:, :H]


@pytest.mark.parametrize("N,H", MANY)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_more_rows_than_run_at_once(N, H, dtype):
    """Each CTA walks several rows, with later ones on their way: every row against the oracle, over the inputs and apart."""
    for pad in (0, 3):
        x, res = random_rows(N, H, dtype, 1, pad), random_rows(N, H, dtype, 2, pad, 2.0)
        w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
        ref = S.rmsnorm_residual_fwd(x, res, w, 0.0, float(torch.tensor(1e-6, dtype=F32)))
        plain = run_fwd(x, res, w, want=("h", "y", "rstd"))
        check_fwd(x, res, w, plain, ref, 0.0, 0)
        for group in (0, 128):
            out = run_fwd(x, res, w, group=group, want=("y", "rstd", "q"))
            assert torch.equal(out["y"], plain["y"]) and torch.equal(out["rstd"], plain["rstd"])
            check_fwd(x, res, w, {k: out[k] for k in ("q", "scales")}, ref, 0.0, group)
        over = run_fwd(x, res, w, want=("rstd",), place={"h": res, "y": x})
        assert torch.equal(over["h"], plain["h"]) and torch.equal(over["y"], plain["y"]) and torch.equal(over["rstd"], plain["rstd"])


@pytest.mark.parametrize("N,H", MANY)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_of_more_rows_than_run_at_once(N, H, dtype):
    for pad in (0, 3):
        dy, dh, h = (random_rows(N, H, dtype, s, pad) for s in (1, 2, 3))
        w = torch.randn(H, generator=torch.Generator().manual_seed(7)).cuda()
        rstd = S.rmsnorm_residual_fwd(h, None, w, 0.0, 1e-6)[1].float().cuda()
        out = run_bwd(dy, dh, h, w, rstd)
        check_bwd(dy, dh, h, w, rstd, out)
        check_bwd(dy, None, h, w, rstd, run_bwd(dy, None, h, w, rstd))
        over = run_bwd(dy, dh, h, w, rstd, dx=dh)
        assert torch.equal(over["dx"], out["dx"]) and torch.equal(over["dw"], out["dw"])


@pytest.mark.parametrize("N,H,dtype", [(13000, 4096, BF16), (50000, 1024, BF16), (12500, 2048, F32), (10000, 5120, BF16), (13001, 4095, BF16)])
def test_large_forward_calls_give_what_their_pieces_give_alone(N, H, dtype):
    """Tensors above 100 MB run with fewer CTAs; pieces of more than 2,048 rows have the same sums, so the same bits."""
    x, res = random_rows(N, H, dtype, 1), random_rows(N, H, dtype, 2, scale=2.0)
    w = torch.randn(H, generator=torch.Generator().manual_seed(7)).to(dtype).cuda()
    np = B.NormParams(1e-6, 1.0, 0, 0)
    h, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(N, device="cuda")
    B.mrl_rmsnorm_residual_fwd(x, res, w, np, h, y, rstd=rstd)
    ph, py, prstd = torch.empty_like(x), torch.empty_like(x), torch.empty(N, device="cuda")
    cuts = list(range(0, N, 2500))[:-1] + [N]
    for lo, hi in zip(cuts, cuts[1:]):
        B.mrl_rmsnorm_residual_fwd(x[lo:hi], res[lo:hi], w, np, ph[lo:hi], py[lo:hi], rstd=prstd[lo:hi])
    torch.cuda.synchronize()
    assert torch.equal(h, ph) and torch.equal(y, py) and torch.equal(rstd, prstd)
    some = slice(N - 40, N)
    ref = S.rmsnorm_residual_fwd(x[some], res[some], w, 1.0, float(torch.tensor(1e-6, dtype=F32)))
    check_fwd(x[some], res[some], w, {"h": h[some], "y": y[some], "rstd": rstd[some]}, ref, 1.0, 0)
    B.mrl_rmsnorm_residual_fwd(x, res, w, np, res, x, rstd=rstd)
    torch.cuda.synchronize()
    assert torch.equal(res, h) and torch.equal(x, y) and torch.equal(rstd, prstd)


@pytest.mark.parametrize("H", [8193, 10007, 12001, 16383])
def test_wide_rows_of_odd_width(H):
    """float32 rows that leave no room for a second row, or for one, in shared memory."""
    for N in (5, 400):
        x, res = random_rows(N, H, F32, 1), random_rows(N, H, F32, 2)
        w = torch.randn(H, generator=torch.Generator().manual_seed(7)).cuda()
        ref = S.rmsnorm_residual_fwd(x, res, w, 0.0, float(torch.tensor(1e-6, dtype=F32)))
        out = run_fwd(x, res, w, group=256, want=("h", "y", "rstd", "q"))
        check_fwd(x, res, w, out, ref, 0.0, 256)
        dy, dh = random_rows(N, H, F32, 3), random_rows(N, H, F32, 4)
        check_bwd(dy, dh, x, w, out["rstd"], run_bwd(dy, dh, x, w, out["rstd"]))
        check_bwd(dy, None, x, w, out["rstd"], run_bwd(dy, None, x, w, out["rstd"]))


def test_gradients_match_differences_of_the_forward_pass():
    """Central differences of sum(y dy) over the float32 forward pass.  Its y are O(1) with an error of (53 / 2 + 10) u each,
    so a sum of 40 products of O(1) is off by 40 * 3 * 37 u = 2.6e-4 at the very most, divided by 2 e = 0.125; the third
    derivative's share, e^2 / 6 times O(10), is 7e-3."""
    H, e = 40, 0.0625
    x, dy = rows(1, H, F32, 1), rows(1, H, F32, 2)
    w = torch.randn(H, generator=torch.Generator().manual_seed(3)).cuda()
    out = run_fwd(x, None, w)
    got = run_bwd(dy, None, x, w, out["rstd"])
    many = x.repeat(2 * H, 1)
    idx = torch.arange(H, device="cuda")
    many[idx, idx] += e
    many[H + idx, idx] -= e
    f = (run_fwd(many, None, w)["y"].double() * dy.double()).sum(1)
    diff = (f[:H] - f[H:]) / (2 * e)
    assert float((diff - got["dx"][0].double()).abs().max()) < 2.1e-3 + 7e-3


def test_forward_and_backward_on_another_stream_and_bitwise_repeatable():
    N, H = 300, 1024
    x, res = rows(N, H, BF16, 1), rows(N, H, BF16, 2)
    w = torch.randn(H, generator=torch.Generator().manual_seed(7)).cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    a = run_fwd(x, res, w, want=("h", "y", "rstd", "q"), group=128)
    b = run_fwd(x, res, w, want=("h", "y", "rstd", "q"), group=128, stream=side)
    for k in ("h", "y", "rstd", "q", "scales"):
        assert torch.equal(a[k], b[k])
    c, d = run_bwd(a["y"], None, a["h"], w, a["rstd"]), run_bwd(a["y"], None, a["h"], w, a["rstd"], stream=side)
    assert torch.equal(c["dx"], d["dx"]) and torch.equal(c["dw"], d["dw"])


def test_binding_refuses_shapes_types_and_strides():
    x, w, np = rows(4, 64, BF16, 1), torch.ones(64, device="cuda"), B.NormParams(1e-6, 0.0, 32, 0)
    y = torch.empty_like(x)
    bad = [dict(residual=rows(3, 64, BF16, 2)), dict(residual=rows(4, 64, F32, 2)), dict(y=rows(4, 128, BF16, 2)[:, ::2]),
           dict(weight=torch.ones(63, device="cuda")), dict(weight=torch.ones(64)), dict(rstd=torch.empty(3, device="cuda")),
           dict(y8=torch.empty(4, 64, dtype=torch.int8, device="cuda"), scales=torch.empty(4, 2, device="cuda")),
           dict(y8=torch.empty(4, 64, dtype=torch.uint8, device="cuda"), scales=torch.empty(4, 1, device="cuda")),
           dict(y8=torch.empty(4, 64, dtype=torch.uint8, device="cuda")), dict(y=x.expand(4, 64)[:1].expand(4, 64))]
    for kw in bad:
        args = dict(x=x, residual=None, weight=w, np=np, y=y) | kw
        with pytest.raises(B.MrlError):
            B.mrl_rmsnorm_residual_fwd(**args)
    with pytest.raises(B.MrlError):
        B.mrl_rmsnorm_residual_bwd(x, None, x, w, torch.ones(4, device="cuda"), B.NormParams(1e-6, 0.0, 0, 0), y, w.clone())
    torch.cuda.synchronize()
