"""The norm's eps below float32's normal range is refused on the host: squares of such rows have no digits left there."""
import pytest

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

FAKE = 0x1000        # never dereferenced: every call below fails validation


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1.1e-38])
def test_norm_refuses_eps_below_the_normal_range(eps):
    build.build()
    np = B.NormParams(eps, 0.0, 0, 0)
    assert 0.0 < np.eps < 2.0 ** -126
    assert B.lib().mrl_rmsnorm_residual_fwd(FAKE, 8, None, 8, B.BF16, FAKE, B.F32, 4, 8, np, None, 8, 0x2000, 8, None, 8, None, None,
                                            None) == 1
