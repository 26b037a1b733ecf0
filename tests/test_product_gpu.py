"""mrl_e4m3_quantize and mrl_e4m3_product against the float64 oracle."""
import math

import pytest
import torch

from oracle import score_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24
E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def quantize(x, rows, pad=0, stride=None):
    N, H = x.shape
    codes = torch.full((N, (stride or H) + pad), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.empty(-(-N // rows), -(-H // 128), device="cuda")
    B.mrl_e4m3_quantize(x, codes[:, :H], scales, rows)
    assert bool((codes[:, H:] == 0x55).all())
    return codes[:, :H], scales


def neighbours(q):
    """The e4m3 values next to a quotient (or the one it is)."""
    grid = torch.arange(256, dtype=torch.uint8).view(E4M3).float()
    grid = grid[grid.isfinite()].unique().double()
    hi = torch.searchsorted(grid, q).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    return grid[lo], grid[hi]


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("N,H,dtype,pad,offset", [
    (1, 1, torch.float32, 0, 0), (3, 127, torch.bfloat16, 1, 1), (129, 128, torch.bfloat16, 0, 0), (130, 260, torch.float32, 3, 1),
    (257, 1003, torch.bfloat16, 5, 3), (300, 4096, torch.bfloat16, 0, 0), (64, 4096, torch.float32, 4, 0), (1000, 136, torch.bfloat16, 8, 8)])
def test_quantize(N, H, dtype, rows, pad, offset):
    g = torch.Generator().manual_seed(N + H)
    flat = torch.full((offset + N * (H + pad) + 8,), 1e6).to(dtype)
    x = flat[offset:offset + N * (H + pad)].view(N, H + pad)[:, :H]
    x.copy_((torch.randn(N, H, generator=g) * torch.exp(torch.randn(H, generator=g)) * 0.02).to(dtype))
    x[0, 0] = 0.0
    if N > 2:
        x[2] = 0.0
    xd = flat.cuda()[offset:].as_strided((N, H), (H + pad, 1))
    for codes_pad in (0, 7):
        codes, scales = quantize(xd, rows, codes_pad)
        peaks = S.block_peaks(x.float(), rows)
        want = (peaks / 448).clamp_min(2.0 ** -126)
        assert bool(((scales.cpu().double() - want).abs() <= 3 * HALF * want).all())       # product with the rounded 1 / 448
        got = codes.cpu().view(E4M3).float().double()
        q = x.double() / S.spread(scales.cpu(), rows, N, H)
        lo, hi = neighbours(q)
        nearest = torch.where((q - lo) <= (hi - q), lo, hi)
        tie = ((q - lo) - (hi - q)).abs() <= 2.0 ** -21 * q.abs()
        assert bool(((got == nearest) | (tie & ((got == lo) | (got == hi)))).all())


def test_quantize_not_finite_and_far():
    x = torch.zeros(4, 400)
    x[0, 5], x[1, 130], x[1, 131] = math.nan, math.inf, 3.0
    x[2, :] = 1e-40
    x[3, 0], x[3, 300] = 3e38, -3e38
    codes, scales = quantize(x.cuda(), 1)
    v, s = codes.cpu().view(E4M3).float(), scales.cpu()
    assert v[0, 5].isnan() and s[0, 0] == 2.0 ** -126 and not v[0, 6:].any()
    assert s[1, 1] == math.inf and v[1, 131] == 0 and v[1, 130].isnan() and s[1, 0] == 2.0 ** -126
    assert bool((s[2] == 2.0 ** -126).all())
    assert v[3, 0] == 448 and v[3, 300] == -448 and s[3].isfinite().all()


def operands(N, H, V, seed, dtype=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x, w = torch.randn(N, H, generator=g), torch.randn(V, H, generator=g) * H ** -0.5
    up = -(-H // 16) * 16
    x8, xs = quantize(x.cuda(), 1, stride=up)
    w8, ws = quantize(w.cuda(), 128, stride=up)
    return x8, xs, w8, ws


def check(out, x8, xs, w8, ws):
    """An element is a sum of H exact products.  Within a block of 128 the tensor core adds four groups of 32 in float32 (cut, not
    rounded: a whole step, 2^-23, each, and as much for aligning a group's products to its largest); the blocks' sums take two
    roundings each for the scale and one for the addition: 2^-23 * (8 + blocks) + 3 * 2^-24 of the sum of magnitudes.  Then one
    rounding to the type."""
    want, size = S.product(x8.cpu().view(E4M3), xs.cpu(), w8.cpu().view(E4M3), ws.cpu())
    tol = size * ((8 + xs.shape[1]) * 2.0 ** -23 + 3 * HALF) + torch.finfo(out.dtype).eps / 2 * want.abs()
    off = (out.cpu().double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol.clamp_min(1e-300)).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,H,V", [(1, 1, 1), (1, 128, 129), (2, 16, 300), (5, 4096, 1000), (17, 130, 255), (64, 256, 256), (65, 384, 700),
                                   (127, 1003, 513), (128, 512, 4096), (200, 1024, 2000), (777, 1003, 5003), (300, 4096, 151), (1, 8192, 40000),
                                   (1000, 640, 777), (16, 1003, 5000), (18, 2048, 20001), (31, 130, 30001), (32, 4096, 19000), (33, 512, 300)])
def test_product(N, H, V, dtype):
    x8, xs, w8, ws = operands(N, H, V, N + H + V)
    wide = torch.full((N + 2, V + 3), 5.0, dtype=dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.mrl_e4m3_product(x8, xs, w8, ws, wide[:N, :V], status)
    torch.cuda.synchronize()
    assert int(status) == 0 and bool((wide[:, V:] == 5.0).all()) and bool((wide[N:] == 5.0).all())
    check(wide[:N, :V], x8, xs, w8, ws)
    again = torch.zeros(N, V, dtype=dtype, device="cuda")
    B.mrl_e4m3_product(x8, xs, w8, ws, again, status)
    assert torch.equal(again, wide[:N, :V])


def test_bytes_between_the_rows_do_not_count():
    x8, xs, w8, ws = operands(40, 100, 200, 1)
    a, b = torch.empty(40, 200, device="cuda"), torch.empty(40, 200, device="cuda")
    B.mrl_e4m3_product(x8, xs, w8, ws, a)
    for t in (x8, w8):
        t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))[:, 100:] = 0x7F          # NaN
    B.mrl_e4m3_product(x8, xs, w8, ws, b)
    assert torch.equal(a, b) and a.isfinite().all()


def test_not_finite_and_far_scales():
    x8, xs, w8, ws = operands(4, 300, 200, 2)
    x8[1, 7] = 0x7F
    xs[2, 1] = 1e30
    ws[1, 2] = 1e-30
    xs[3, 0] = math.inf
    out = torch.empty(4, 200, device="cuda")
    B.mrl_e4m3_product(x8, xs, w8, ws, out)
    assert out[1].isnan().all() and out[0].isfinite().all() and not out[3].isfinite().any()
    check(out[[0, 2]], x8[[0, 2]], xs[[0, 2]], w8, ws)


def test_one_hot_rows_give_the_weights_back():
    """Which element meets which: row t picks column c_t, so the output is w[v, c_t] exactly."""
    H, V = 700, 900
    c = torch.randperm(H)[:300]
    x8 = torch.zeros(300, 704, dtype=torch.uint8)
    x8[torch.arange(300), c] = 0x38                        # 1.0
    w8 = torch.randint(0, 0x7E, (V, 704), dtype=torch.uint8)
    one = lambda n: torch.ones(n, 6, device="cuda")  # noqa: E731
    out = torch.empty(300, V, device="cuda")
    B.mrl_e4m3_product(x8.cuda()[:, :H], one(300), w8.cuda()[:, :H], one(8), out)
    assert torch.equal(out.cpu(), w8.view(E4M3).float()[:, c].T)


def test_large_rows_and_a_side_stream():
    """Output offsets that pass 32 bits, on a stream of its own, from a graph."""
    N, H, V = 17000, 128, 151936
    x8, xs, w8, ws = operands(N, H, V, 3)
    out = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.mrl_e4m3_product(x8, xs, w8, ws, out, stream=side)
    graph.replay()
    torch.cuda.synchronize()
    pick = torch.tensor([0, 1, 8191, 14132, 14133, 16999])
    check(out[pick.cuda()], x8[pick.cuda()], xs[pick.cuda()], w8, ws)
    assert int((out == 0).sum(dtype=torch.int64)) < N * V // 1000
