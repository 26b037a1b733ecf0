"""The 8-bit product where the product of two scales is at an end of float32's normal range, for few rows and for many."""
import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

import test_product_gpu as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()
    B.lib()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [4, 24, 40, 200])
def test_smallest_products_of_scales(N, dtype):
    """2^-126 for each block, from both sides; and blocks of zeros, whose scale is 2^-126 by itself, beside ordinary ones."""
    x8, xs, w8, ws = P.operands(N, 300, 200, N)
    for ex, ew in ((-63, -63), (-126, 0), (0, -126), (-100, -26)):
        a, b = torch.full_like(xs, 2.0 ** ex), torch.full_like(ws, 2.0 ** ew)
        out = torch.empty(N, 200, dtype=dtype, device="cuda")
        B.mrl_e4m3_product(x8, a, w8, b, out)
        P.check(out, x8, a, w8, b)
    x8[:, 128:256] = 0
    xs[:, 1] = 2.0 ** -126
    ws[:, 1] = 2.0 ** -40
    out = torch.empty(N, 200, dtype=dtype, device="cuda")
    B.mrl_e4m3_product(x8, xs, w8, ws, out)
    P.check(out, x8, xs, w8, ws)


@pytest.mark.parametrize("N", [4, 24, 40, 200])
def test_largest_products_of_scales(N):
    """2^127: rows of one code 2^-9 pick single weights, so that nothing is rounded and nothing leaves float32."""
    H, V = 300, 200
    c = torch.randperm(H)[:N]
    x8 = torch.zeros(N, 304, dtype=torch.uint8)
    x8[torch.arange(N), c] = 0x01
    w8 = torch.randint(0, 0x7E, (V, 304), dtype=torch.uint8)
    for ex, ew in ((63, 64), (127, 0), (0, 127)):
        out = torch.empty(N, V, device="cuda")
        B.mrl_e4m3_product(x8.cuda()[:, :H], torch.full((N, 3), 2.0 ** ex, device="cuda"), w8.cuda()[:, :H],
                           torch.full((2, 3), 2.0 ** ew, device="cuda"), out)
        want = w8.view(torch.float8_e4m3fn).double()[:, c].T * 2.0 ** 118
        assert torch.equal(out.cpu().double(), want)
