"""Addresses that are not on an element are refused on the host: on the device they would be a misaligned access."""
import pytest

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

FAKE = 0x1000        # never dereferenced: every call below fails validation


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def slot(**kw):
    base = dict(grad=FAKE, param=0x2000, master=None, m=0x3000, v=0x4000, m_scale=None, v_scale=None, numel=10, rng_first=0,
                weight_decay=0.0, grad_dtype=B.F32, param_dtype=B.F32, state_dtype=B.F32)
    return B.TensorSlotStruct(**(base | kw))


def table(*slots):
    return (B.TensorSlotStruct * len(slots))(*slots)


@pytest.mark.parametrize("bad", [
    dict(grad=FAKE + 2), dict(grad=FAKE + 1, grad_dtype=B.BF16), dict(param=0x2002), dict(param=0x2001, param_dtype=B.BF16),
    dict(param_dtype=B.BF16, master=0x5002), dict(m=0x3001), dict(v=0x4002),
    dict(state_dtype=B.E4M3, m=0x3001, v=0x4003, m_scale=0x6002, v_scale=0x7000),
    dict(state_dtype=B.E4M3, m_scale=0x6000, v_scale=0x7001)])
def test_adamw_refuses_tensors_off_their_elements(lib, bad):
    ap = B.AdamwParams(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    assert lib.mrl_adamw_step(table(slot(), slot(**bad)), 2, ap, None, None, None, 0, None) == 1


@pytest.mark.parametrize("kw", [dict(grad_scale=FAKE + 2), dict(status=FAKE + 1), dict(lr_dev=FAKE + 2), dict(step_dev=FAKE + 4)])
@pytest.mark.parametrize("n", [0, 1])
def test_adamw_refuses_scalars_off_their_elements(lib, kw, n):
    ap = B.AdamwParams(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, lr_dev=kw.get("lr_dev"), step_dev=kw.get("step_dev"))
    assert lib.mrl_adamw_step(table(slot()), n, ap, kw.get("grad_scale"), kw.get("status"), FAKE, 512, None) == 1


def test_grad_norm_refuses_addresses_off_their_elements(lib):
    def call(s=slot(), norm=FAKE, coef=FAKE):
        return lib.mrl_grad_norm(table(slot(), s), 2, 1.0, norm, coef, FAKE, 1 << 20, None)

    assert call(slot(grad=FAKE + 2)) == 1 and call(slot(grad=FAKE + 1, grad_dtype=B.BF16)) == 1
    assert call(norm=FAKE + 2) == 1 and call(coef=FAKE + 1) == 1


def test_norm_refuses_float32_vectors_off_their_elements(lib):
    np = B.NormParams(1e-6, 0.0, 0, 0)

    def fwd(scales=FAKE, rstd=FAKE):
        return lib.mrl_rmsnorm_residual_fwd(FAKE, 8, None, 8, B.BF16, FAKE, B.F32, 4, 8, np, None, 8, None, 8, 0x2001, 8,
                                            scales, rstd, None)

    def bwd(rstd=FAKE, dw=FAKE):
        return lib.mrl_rmsnorm_residual_bwd(FAKE, 8, None, 8, FAKE, 8, B.F32, FAKE, B.F32, rstd, 4, 8, np, FAKE, 8, dw, FAKE,
                                            1 << 20, None)

    assert fwd(scales=FAKE + 2) == 1 and fwd(rstd=FAKE + 1) == 1
    assert bwd(rstd=FAKE + 2) == 1 and bwd(dw=FAKE + 3) == 1
