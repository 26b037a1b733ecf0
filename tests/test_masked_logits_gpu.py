"""Top tokens and distillation where logits z c, c = log2(e) / T, are too large for float32 to hold the steps between them: masks of -1e9, -1e10, -1e30 and of the
type's lowest value at several temperatures, logits of that size, and temperatures that make ordinary logits so large.

Between magnitudes of 2^24 and 2^31 of z c the offset that a row's exponents are taken against is a float, so up to 64 off the largest of them (half a step below
2^31).  That offset is in the sum as a factor of 2^64 at most and comes out again as ln s: `OFFSET`, 64 ln 2 < 45, is a magnitude that log-probs and entropies are
differences of there, besides those that test_top_gpu.py counts."""
import math

import pytest
import torch

from oracle import score_oracle as S
from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

import test_distill_gpu as D
import test_top_gpu as U

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24
OFFSET = 45.0
KINDS = sorted(D.KINDS)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


def fills(dtype):
    return [-1e9, -1e10, -1e30, torch.finfo(dtype).min, 0.5 * torch.finfo(dtype).min]


def masked_rows(V, dtype):
    """For each mask: a tail of the vocabulary, the first token, the last, stretches of a few thousand, all but one token, all."""
    g = torch.Generator().manual_seed(V)
    out = []
    for fill in fills(dtype):
        for kind in range(6):
            z = torch.randn(V, generator=g) * 2.0
            v = torch.arange(V)
            z[[v >= V - V // 5, v == 0, v == V - 1, v // 3000 % 2 == 1, v != V // 3, v >= 0][kind]] = fill
            out.append(z)
    return torch.stack(out).to(dtype)


def large_rows(V, dtype):
    """Logits that are themselves that large."""
    g = torch.Generator().manual_seed(V + 2)
    r = lambda: torch.randn(V, generator=g)  # noqa: E731
    one = lambda x: torch.where(torch.arange(V) == V // 2, torch.tensor(x), r())  # noqa: E731
    top = torch.finfo(dtype).max
    return torch.stack([one(1e10), one(1e30), one(top), torch.full((V,), top), torch.full((V,), 1e10), r() * 1e12, r() * 1e36, r() * 1e9 - 4e9]).to(dtype)


def check_top(z, got, ids, T, top):
    V = z.shape[1]
    lse, logp, entropy, lists, top_logp = S.top_logprobs(z.float(), ids, T, top)
    base = U.chain(V) + (4 + 4 * OFFSET) * HALF
    assert torch.equal(got["ids"], lists)
    for name, a, b, tol in (("lse", got["lse"], lse, base + 4 * HALF * lse.abs()), ("logp", got["logp"], logp, base + 4 * HALF * logp.abs()),
                            ("top", got["top"], top_logp, base + 4 * HALF * top_logp.abs()),
                            ("entropy", got["entropy"], entropy, 2 * base * torch.full_like(lse, 1 + math.log(V) + OFFSET))):
        far = b.abs() > torch.finfo(torch.float32).max          # (a log-prob that float32 cannot hold)
        fine = torch.where(far, a == torch.where(b > 0, math.inf, -math.inf), (a - b).abs() <= tol)
        assert bool(fine.all()), (name, (~fine).nonzero()[:5].tolist(), a[~fine][:5].tolist(), b[~fine][:5].tolist())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [0.7, 1.0, 1.5, 2.0, 2.5, 4.0])
@pytest.mark.parametrize("V,top,N", [(1003, 20, 800), (2722, 20, 0), (6007, 40, 760), (40001, 128, 0), (70003, 20, 420)])
def test_top_tokens_of_masked_and_large_rows(V, top, N, T, dtype):
    z = torch.cat([masked_rows(V, dtype), large_rows(V, dtype)])
    n = z.shape[0]
    if N:       # (many rows are worked on by other kernels than few)
        z = torch.cat([z, U.rows(N - n, V, dtype, V)[0]])
    ids = torch.randint(0, V, (z.shape[0],), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    T = float(torch.tensor(T))
    got = U.run(z, z.reshape(-1), ids, None, T, top)
    assert got["status"] == 0
    check_top(z[:n], {k: v[:n] if torch.is_tensor(v) else v for k, v in got.items()}, ids[:n], T, top)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1e-6, 1e-4, 0.01, 1e6])
def test_top_tokens_at_far_temperatures(T, dtype):
    V = 5003
    g = torch.Generator().manual_seed(3)
    z = torch.stack([torch.randn(V, generator=g) * 2 + shift for shift in (0.0, 2000.0, -2000.0, 1e5, -1e5)]).to(dtype)
    ids = torch.randint(0, V, (5,), generator=g, dtype=torch.int32)
    T = float(torch.tensor(T))
    check_top(z, U.run(z, z.reshape(-1), ids, None, T, 20), ids, T, 20)


def test_not_finite_rows_stay_so_beside_large_logits():
    V = 9001
    z = torch.randn(6, V, generator=torch.Generator().manual_seed(1))
    z[0, 5], z[1, 7], z[1, 9], z[2], z[3, 8000], z[4, 4] = math.nan, math.nan, 1e30, math.inf, math.inf, -math.inf
    z[3, 3] = 1e30
    got = U.run(z, z.reshape(-1), torch.zeros(6, dtype=torch.int32), None, 1.0, 5)
    assert got["lse"][:4].isnan().all() and got["entropy"][:4].isnan().all() and got["lse"][4:].isfinite().all()


def masked_lists(V, top, dtype, N):
    """Rows with a list each; the masks of masked_rows in the other tokens, then all other tokens, the whole row, and the listed tokens alone."""
    g = torch.Generator().manual_seed(V + top)
    rows, v = [], torch.arange(V)
    ids = torch.stack([torch.randperm(V, generator=g)[:top] for _ in range(max(N, 8 * 5))]).int()
    for fill in fills(dtype):
        for kind in range(8):
            z = torch.randn(V, generator=g) * 2.0
            listed = torch.zeros(V, dtype=torch.bool)
            listed[ids[len(rows)].long()] = True
            free = (~listed).nonzero()[:, 0]
            where = [(v >= V - V // 5) & ~listed, v == free[0], v == free[-1], (v // 3000 % 2 == 1) & ~listed, ~listed & (v != free[7]), ~listed,
                     v >= 0, listed][kind]
            if kind == 7 and fill < -1e31:      # (its KL, q times |fill| / T, could leave float32)
                fill = -1e30
            z[where] = fill
            rows.append(z)
    z = torch.stack(rows + [torch.randn(V, generator=g) * 2.0 for _ in range(len(ids) - len(rows))]).to(dtype)
    logq = torch.log_softmax(torch.randn(len(ids), top + 1, generator=g), 1)[:, :top].contiguous()
    return z, ids, logq


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [0.7, 1.0, 1.5, 2.0, 2.5, 4.0])
@pytest.mark.parametrize("V,top,N", [(1003, 20, 420), (5000, 8, 0), (100003, 20, 0)])
def test_distillation_of_masked_rows(V, top, N, T, kind, dtype):
    z, ids, logq = masked_lists(V, top, dtype, N)
    dp = D.params(kind, float(torch.tensor(T)), 0.7)
    got = D.run(z, z.reshape(-1), ids, logq, None, None, dp)
    assert got["row_kl"].isfinite().all() and got["dz"].isfinite().all() and math.isfinite(got["loss"])
    D.check(z, got, ids, logq, None, None, dp)
    again = D.run(z, z.reshape(-1), ids, logq, None, None, dp, in_place=True)
    assert torch.equal(got["dz"].view(torch.uint8), again["dz"].view(torch.uint8)) and torch.equal(got["row_kl"], again["row_kl"])
