"""An output over an input with another row stride would overwrite rows that are still to be read: refused on the host."""
import pytest

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

FAKE = 0x1000        # never dereferenced: every call below fails validation


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def fwd(lib, N=4, x=0x1000, ld_x=16, res=0x2000, ld_res=24, h=None, ld_h=8, y=None, ld_y=8, y8=None):
    np = B.NormParams(1e-6, 0.0, 0, 0)
    return lib.mrl_rmsnorm_residual_fwd(x, ld_x, res, ld_res, B.BF16, 0x9000, B.F32, N, 8, np, h, ld_h, y, ld_y, y8, 8, 0x7000,
                                        0x8000, None)


@pytest.mark.parametrize("kw", [dict(h=0x1000, ld_h=8), dict(h=0x2000, ld_h=16), dict(y=0x1000, ld_y=24), dict(y=0x2000, ld_y=8),
                                dict(y8=0x1000), dict(y8=0x2000), dict(h=0x3000, y8=0x3000), dict(y=0x3000, y8=0x3000)])
def test_forward_refuses(lib, kw):
    assert fwd(lib, **kw) == 1


@pytest.mark.parametrize("kw", [dict(dx=0x1000, ld_dx=8), dict(dx=0x2000, ld_dx=16), dict(dx=0x3000, ld_dx=16)])
def test_backward_refuses(lib, kw):
    np = B.NormParams(1e-6, 0.0, 0, 0)
    assert lib.mrl_rmsnorm_residual_bwd(0x1000, 16, 0x2000, 24, 0x3000, 8, B.BF16, 0x9000, B.F32, 0x8000, 4, 8, np, kw["dx"],
                                        kw["ld_dx"], None, None, 0, None) == 1
