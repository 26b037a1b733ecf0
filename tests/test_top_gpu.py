"""mrl_top_logprobs against the float64 oracle: ids exactly, the rest within the roundings of the sums.

A row's sum takes at most V / 256 + 64 additions one after the other, each off by half a step (2^-24) of the sum, over terms off by
at most 2^-22 (exponential) + 2^-23 |t| (its argument; |t| 2^t < 1): `chain` below.  The results are rounded once more, relative to
themselves and to lse."""
import math

import pytest
import torch

from oracle import score_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def chain(V):
    return (V / 256 + 64 + 8) * HALF


def rows(N, V, dtype, seed, pad=0, offset=0, scale=2.0):
    """[N, V] rows in a wider buffer that starts `offset` elements behind a 256-byte boundary."""
    g = torch.Generator().manual_seed(seed)
    flat = torch.full((offset + N * (V + pad) + 8,), 1e4).to(dtype)          # what lies between the rows would top every list
    z = flat[offset:offset + N * (V + pad)].view(N, V + pad)[:, :V]
    z.copy_((torch.randn(N, V, generator=g) * scale).to(dtype))
    return z, flat


def run(z, flat, ids, mask, T, top, stream=None):
    N, V = z.shape
    dev = flat.cuda()
    zd = dev[z.storage_offset():].as_strided((N, V), (z.stride(0), 1)) if N else dev[:0].view(0, V)
    guard = 16
    out = {k: torch.full((N + guard,), 7.25, device="cuda") for k in ("logp", "lse", "entropy")}
    tops = torch.full((N + guard, top), 77, dtype=torch.int32, device="cuda"), torch.full((N + guard, top), 7.25, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cut = {k: v[:N] for k, v in out.items()}
    if ids is None:
        cut["logp"] = None
    B.mrl_top_logprobs(zd, None if ids is None else ids.cuda(), None if mask is None else mask.cuda(), T, cut["logp"], cut["lse"],
                       cut["entropy"], tops[0][:N] if top else None, tops[1][:N] if top else None, status, stream=stream)
    torch.cuda.synchronize()
    for v in out.values():
        assert bool((v[N:] == 7.25).all())
    assert bool((tops[0][N:] == 77).all()) and bool((tops[1][N:] == 7.25).all())
    got = {k: v[:N].cpu().double() for k, v in out.items()}
    return got | {"ids": tops[0][:N].cpu().long(), "top": tops[1][:N].cpu().double(), "status": int(status)}


def check(z, got, ids, mask, T, top):
    V = z.shape[1]
    lse, logp, entropy, lists, top_logp = S.top_logprobs(z.float(), ids, T, top)
    on = torch.ones(z.shape[0], dtype=torch.bool) if mask is None else mask.bool()
    assert torch.equal(got["ids"][on], lists[on])
    assert bool((got["ids"][~on] == -1).all()) and not bool(got["top"][~on].any()) and not bool(got["lse"][~on].any())

    def near(a, b, tol):
        a, b, tol = a[on], b[on], tol[on]
        same = (a == b) | (a.isnan() & b.isnan())
        assert bool((same | ((a - b).abs() <= tol)).all()), float(((a - b).abs() - tol)[~same].max())

    size = lse.abs().nan_to_num(0.0)
    base = chain(V) + 4 * HALF
    near(got["lse"], lse, base + 4 * HALF * size)
    if ids is not None:
        near(got["logp"], logp, base + 4 * HALF * logp.abs().nan_to_num(0.0, 0.0, 0.0))
    near(got["top"], top_logp, base + 4 * HALF * top_logp.abs().nan_to_num(0.0, 0.0, 0.0))
    near(got["entropy"], entropy, (2 * base + 2 * HALF * 32) * torch.full_like(lse, 1 + math.log(V)))   # |t| < 32 where 2^t t counts


@pytest.mark.parametrize("N,V,dtype,top,T,pad,offset", [
    (1, 1, torch.float32, 1, 1.0, 0, 0), (3, 2, torch.bfloat16, 2, 2.0, 0, 1), (5, 33, torch.bfloat16, 7, 0.7, 3, 3),
    (4, 129, torch.float32, 128, 1.0, 0, 1), (7, 1000, torch.bfloat16, 20, 1.0, 0, 0), (2, 4096, torch.float32, 1, 1.0, 8, 0),
    (9, 8191, torch.bfloat16, 128, 1.0, 1, 5), (3, 16385, torch.float32, 64, 0.5, 2, 3), (2, 32003, torch.bfloat16, 0, 1.0, 0, 0),
    (1, 151936, torch.bfloat16, 20, 1.0, 0, 0), (3, 151936, torch.float32, 128, 1.0, 0, 0), (2, 128257, torch.bfloat16, 64, 1.3, 6, 7),
    (400, 5003, torch.bfloat16, 50, 1.0, 5, 1), (700, 4096, torch.float32, 5, 1.0, 0, 0), (310, 40000, torch.bfloat16, 128, 1.0, 0, 0),
])
def test_rows_of_all_sizes(N, V, dtype, top, T, pad, offset):
    z, flat = rows(N, V, dtype, N + V, pad, offset)
    g = torch.Generator().manual_seed(5)
    ids = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    mask = (torch.rand(N, generator=g) < 0.8).to(torch.uint8) if N > 3 else None
    got = run(z, flat, ids, mask, float(torch.tensor(T)), top)
    assert got["status"] == 0
    check(z, got, ids, mask, float(torch.tensor(T)), top)


def special_rows(V, dtype, N):
    """Rows where threshold, order or arithmetic can go wrong."""
    g = torch.Generator().manual_seed(V)
    low = torch.finfo(dtype).min
    r = lambda: torch.randn(V, generator=g)  # noqa: E731
    few = torch.full((V,), -math.inf)
    few[torch.randperm(V, generator=g)[:3]] = 1.0
    late = torch.full((V,), -math.inf)
    late[-5:] = torch.tensor([1.0, 2.0, 2.0, 0.5, 3.0])[:min(5, V)] if V >= 5 else 1.0
    ends = torch.full((V,), low)
    ends[0], ends[-1] = 2.0, 2.0
    steps = torch.arange(V).float() / V
    nans = r()
    nans[V // 2] = math.nan
    inf = r()
    inf[V // 3] = math.inf
    mixed = r()
    mixed[torch.rand(V, generator=g) < 0.9] = low
    half = torch.cat([torch.full((V - V // 2,), -math.inf), r()[:V // 2]])
    far = torch.zeros(V)
    far[V - 1] = 1e30
    out = [torch.zeros(V), torch.full((V,), -math.inf), torch.full((V,), low), few, late, ends, steps, -steps, torch.full((V,), math.nan),
           nans, inf, mixed, half, far, (r() * 3).round(), torch.cat([r()[:V // 2] - 50, r()[:V - V // 2] + 50]), -torch.zeros(V)]
    out = out + [r() for _ in range(max(0, N - len(out)))]
    return torch.stack(out).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,top,N", [(7, 7, 0), (300, 128, 0), (5000, 20, 0), (40001, 128, 0), (151936, 3, 0), (20011, 40, 310), (150000, 128, 310)])
def test_special_rows(dtype, V, top, N):
    z = special_rows(V, dtype, N)
    assert z.shape[0] < 296 or N       # few rows are cut among CTAs, many are not
    got = run(z, z.view(-1), None, None, 1.0, top)
    check(z[:17], {k: v[:17] if torch.is_tensor(v) else v for k, v in got.items()}, None, None, 1.0, top)
    if N:
        check(z[-3:], {k: v[-3:] if torch.is_tensor(v) else v for k, v in got.items()}, None, None, 1.0, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,top,N", [(40, 32, 800), (1003, 32, 900), (1003, 64, 900), (2722, 4, 1500), (3001, 33, 760), (9001, 64, 790), (24001, 20, 745),
                                     (32768, 64, 741), (3000, 128, 800)])
def test_short_rows_of_many(V, top, N, dtype):
    """More rows than are worked on at a time: special, crowded and plain ones, with bad ids and masked rows among them."""
    z = torch.cat([special_rows(V, dtype, 0), crowded_rows(V, dtype, 0), rows(N - 27, V, dtype, V)[0]])
    ids = torch.randint(0, V, (N,), generator=torch.Generator().manual_seed(2), dtype=torch.int32)
    mask = torch.ones(N, dtype=torch.uint8)
    ids[40], ids[50], mask[60], mask[61], ids[61] = V, -1, 0, 0, V
    got = run(z, z.reshape(-1), ids, mask, 1.0, top)
    assert got["status"] == B.DEV_BAD_TOKEN_ID
    fine = torch.ones(N, dtype=torch.bool)
    fine[[40, 50, 60, 61]] = False
    check(z[fine], {k: v[fine] if torch.is_tensor(v) else v for k, v in got.items()}, ids[fine], mask[fine], 1.0, top)
    for k in ("logp", "lse", "entropy", "top"):
        assert not bool(got[k][~fine].any())


def crowded_rows(V, dtype, N):
    """Rows where more tokens than a list of candidates holds are near its last place."""
    g = torch.Generator().manual_seed(V + 1)
    low = torch.finfo(dtype).min
    rising = torch.arange(V).float() * 2.0 ** -14
    ten = torch.full((V,), low)
    ten[torch.randperm(V, generator=g)[:10]] = torch.randn(10, generator=g)
    few_values = torch.randint(-2, 3, (V,), generator=g).float()
    crowd = torch.where(torch.rand(V, generator=g) < 0.7, torch.tensor(0.5), torch.randn(V, generator=g) * 0.2)
    bands = torch.randn(V, generator=g) + torch.where((torch.arange(V) // 8) % 256 < 150, 100.0, 0.0)
    signs = torch.where(torch.rand(V, generator=g) < 0.5, torch.tensor(-0.0), torch.tensor(0.0))
    below = -1.0 - torch.rand(V, generator=g) * 2.0 ** -6
    out = [rising, -rising, rising.flip(0) * 3, ten, few_values, crowd, bands, signs, below, -few_values.abs()]
    return torch.stack(out + [torch.randn(V, generator=g) for _ in range(max(0, N - len(out)))]).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V,top,N", [(40001, 128, 0), (151936, 20, 0), (151936, 128, 310), (20011, 100, 310)])
def test_crowded_rows(dtype, V, top, N):
    z = crowded_rows(V, dtype, N)
    got = run(z, z.view(-1), None, None, 1.0, top)
    check(z[:10], {k: v[:10] if torch.is_tensor(v) else v for k, v in got.items()}, None, None, 1.0, top)


def test_bad_ids_and_masks():
    z, flat = rows(6, 5000, torch.bfloat16, 1)
    ids = torch.tensor([0, -1, 4999, 5000, 7, 2 ** 31 - 1], dtype=torch.int32)
    got = run(z, flat, ids, None, 1.0, 4)
    assert got["status"] == B.DEV_BAD_TOKEN_ID
    check(z[[0, 2, 4]], {k: v[[0, 2, 4]] if torch.is_tensor(v) else v for k, v in got.items()}, ids[[0, 2, 4]], None, 1.0, 4)
    for k in ("logp", "lse", "entropy", "top"):
        assert not bool(got[k][[1, 3, 5]].any())
    assert bool((got["ids"][[1, 3, 5]] == -1).all())
    off = torch.tensor([0, 0, 1, 0, 0, 0], dtype=torch.uint8)
    got = run(z, flat, ids, off, 1.0, 4)            # the bad ids stand in masked rows
    assert got["status"] == 0
    check(z, got, ids.clamp(0, 4999), off, 1.0, 4)
    assert run(z, flat, ids, torch.zeros(6, dtype=torch.uint8), 1.0, 4)["status"] == 0
    run(z[:0], flat, ids[:0], None, 1.0, 4)


def test_logp_is_that_of_token_logprobs_and_calls_repeat():
    z, flat = rows(500, 32000, torch.bfloat16, 3)
    ids = torch.randint(0, 32000, (500,), dtype=torch.int32)
    a, b = run(z, flat, ids, None, 1.0, 20), run(z, flat, ids, None, 1.0, 20)
    for k in ("logp", "lse", "entropy", "ids", "top"):
        assert torch.equal(a[k], b[k]), k
    logp = torch.empty(500, device="cuda")
    B.mrl_token_logprobs(z.cuda().contiguous(), ids.cuda(), None, logp)
    assert float((logp.cpu().double() - a["logp"]).abs().max()) < 1e-4


def test_rows_past_four_gigabytes():
    """Offsets in elements that pass 32 bits."""
    N, V = 34000, 70000
    z = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    at = torch.randint(0, V, (N,), device="cuda")
    z.scatter_(1, at[:, None], 5.0)
    ids, top, lse = torch.empty(N, 2, dtype=torch.int32, device="cuda"), torch.empty(N, 2, device="cuda"), torch.empty(N, device="cuda")
    B.mrl_top_logprobs(z, None, None, 1.0, None, lse, None, ids, top)
    assert torch.equal(ids[:, 0].long(), at) and torch.equal(ids[:, 1].long(), (at == 0).long())
    want = math.log(math.exp(5.0) + V - 1)
    assert float((lse.double() - want).abs().max()) < chain(V) + 8 * HALF * want
    del z


def test_side_stream_and_graph():
    z, flat = rows(64, 50000, torch.bfloat16, 9)
    ids = torch.randint(0, 50000, (64,), dtype=torch.int32).cuda()
    zd = z.cuda().contiguous()
    make = lambda: [torch.zeros(64, device="cuda"), torch.zeros(64, 30, dtype=torch.int32, device="cuda"), torch.zeros(64, 30, device="cuda")]  # noqa: E731
    a, b = make(), make()
    call = lambda o, st: B.mrl_top_logprobs(zd, ids, None, 1.0, o[0], None, None, o[1], o[2], stream=st)  # noqa: E731
    call(a, None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(b, side)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    zd.neg_()
    call(a, None)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
