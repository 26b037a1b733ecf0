"""What the norm, gradient norm and update entry points refuse, on the host before a device is touched."""
import ctypes as C

import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

FAKE = 0x1000        # never dereferenced: every call below fails validation or is a no-op


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def test_workspace_sizes(lib):
    a, b = B.workspace_bytes(B.WS_RMSNORM_BWD, 10, 0, 100), B.workspace_bytes(B.WS_RMSNORM_BWD, 100000, 0, 4096)
    assert 0 < a < b and a % 256 == 0 and b % 256 == 0
    assert B.workspace_bytes(B.WS_RMSNORM_BWD, 0, 0, 100) == 0 and B.workspace_bytes(B.WS_RMSNORM_BWD, 5, 0, 0) == 0
    assert B.workspace_bytes(B.WS_GRAD_NORM, 0, 0) % 256 == 0 < B.workspace_bytes(B.WS_GRAD_NORM, 0, 0)
    assert B.workspace_bytes(B.WS_ADAMW, 0, 0) > 0


def test_rmsnorm_fwd_refusals(lib):
    def call(x=FAKE, ld_x=8, res=None, ld_res=8, dtype=B.BF16, w=FAKE, wt=B.F32, N=4, H=8, eps=1e-6, off=0.0, group=0,
             h=None, ld_h=8, y=FAKE, ld_y=8, y8=None, ld8=8, scales=None, rstd=None, np=True):
        p = B.NormParams(eps, off, group, 0)
        return lib.mrl_rmsnorm_residual_fwd(x, ld_x, res, ld_res, dtype, w, wt, N, H, p if np else None, h, ld_h, y, ld_y,
                                            y8, ld8, scales, rstd, None)

    assert call(np=False) == 1 and call(N=-1) == 1 and call(H=0) == 1
    assert call(dtype=B.E4M3) == 3 and call(wt=7) == 3
    assert call(eps=0.0) == 1 and call(eps=float("nan")) == 1 and call(eps=float("inf")) == 1 and call(off=float("inf")) == 1
    assert call(group=16) == 1 and call(group=-1) == 1 and call(group=512) == 1
    assert call(ld_x=7) == 1 and call(res=FAKE, ld_res=7) == 1 and call(ld_y=7) == 1 and call(h=0x2000, ld_h=7) == 1
    assert call(y8=FAKE) == 1 and call(y8=FAKE, scales=FAKE, ld8=7) == 1          # codes without scales; a short row
    assert call(y=None) == 1 and call(h=0x3000, y=0x3000) == 1                     # no output; one buffer for two
    assert call(x=None) == 1 and call(w=None) == 1
    assert call(x=0x1001) == 1 and call(w=0x1002) == 1 and call(y=0x1001) == 1 and call(h=0x2001) == 1    # not on an element
    big = (1 << 30) + 1
    assert call(H=big, ld_x=big, ld_y=big) == 7
    assert call(x=None, N=0) == 0


def test_rmsnorm_bwd_refusals(lib):
    def call(dy=FAKE, ld_dy=8, dh=None, ld_dh=8, h=FAKE, ld_h=8, dtype=B.F32, w=FAKE, wt=B.F32, rstd=FAKE, N=4, H=8,
             off=0.0, flags=0, dx=FAKE, ld_dx=8, dw=FAKE, ws=FAKE, ws_bytes=1 << 20, np=True):
        p = B.NormParams(1e-6, off, 0, flags)
        return lib.mrl_rmsnorm_residual_bwd(dy, ld_dy, dh, ld_dh, h, ld_h, dtype, w, wt, rstd, N, H, p if np else None, dx,
                                            ld_dx, dw, ws, ws_bytes, None)

    assert call(np=False) == 1 and call(N=-1) == 1 and call(H=0) == 1 and call(flags=1) == 1 and call(off=float("nan")) == 1
    assert call(dtype=2) == 3 and call(wt=2) == 3
    assert call(ld_dy=7) == 1 and call(ld_h=7) == 1 and call(ld_dx=7) == 1 and call(dh=FAKE, ld_dh=7) == 1
    assert call(dy=None) == 1 and call(h=None) == 1 and call(rstd=None) == 1 and call(dx=None) == 1 and call(w=None) == 1
    assert call(ws=None) == 4 and call(ws_bytes=16) == 4 and call(ws=0x1010) == 1
    assert call(dy=0x1002) == 1 and call(dh=0x1001) == 1 and call(h=0x1003) == 1 and call(dx=0x1002) == 1
    big = (1 << 30) + 1
    assert call(H=big, ld_dy=big, ld_h=big, ld_dx=big) == 7
    assert call(N=0, dw=None) == 0


def slot(**kw):
    base = dict(grad=FAKE, param=FAKE, master=None, m=FAKE, v=FAKE, m_scale=None, v_scale=None, numel=10, rng_first=0,
                weight_decay=0.0, grad_dtype=B.F32, param_dtype=B.F32, state_dtype=B.F32)
    return B.TensorSlotStruct(**(base | kw))


def test_grad_norm_refusals(lib):
    def call(slots=(slot(),), n=None, max_norm=1.0, norm=FAKE, coef=FAKE, ws=FAKE, ws_bytes=1 << 20):
        arr = (B.TensorSlotStruct * len(slots))(*slots) if slots is not None else None
        return lib.mrl_grad_norm(arr, len(slots) if n is None else n, max_norm, norm, coef, ws, ws_bytes, None)

    assert call(n=-1) == 1 and call(slots=None, n=1) == 1 and call(max_norm=float("nan")) == 1
    assert call(norm=None, coef=None) == 1
    assert call((slot(grad=None),)) == 1 and call((slot(numel=-1),)) == 1 and call((slot(), slot(numel=1 << 60),)) == 1
    assert call((slot(grad_dtype=B.E4M3),)) == 3
    assert call(ws=None) == 4 and call(ws_bytes=8) == 4 and call(ws=0x1010) == 1


def test_adamw_refusals(lib):
    def call(slots=(slot(),), n=None, ap=None, ws=None, ws_bytes=0, **kw):
        base = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0, rounding=0, flags=0)
        p = B.AdamwParams(**(base | kw))
        arr = (B.TensorSlotStruct * len(slots))(*slots) if slots is not None else None
        return lib.mrl_adamw_step(arr, len(slots) if n is None else n, p if ap is None else None, None, None, ws, ws_bytes, None)

    assert call(ap=0) == 1 and call(n=-1) == 1 and call(slots=None, n=1) == 1
    assert call(beta1=1.0) == 1 and call(beta1=-0.1) == 1 and call(beta2=float("nan")) == 1
    assert call(eps=0.0) == 1 and call(eps=1e-60) == 1 and call(eps=1e-40) == 1 and call(eps=float("inf")) == 1 and call(lr=float("nan")) == 1
    assert call(step=0) == 1 and call(rounding=2) == 1 and call(flags=1) == 1
    for bad in (dict(grad=None), dict(param=None), dict(m=None), dict(v=None), dict(numel=-1), dict(master=FAKE),
                dict(weight_decay=float("inf")), dict(state_dtype=B.E4M3), dict(state_dtype=B.E4M3, m_scale=FAKE)):
        assert call((slot(), slot(**bad))) == 1, bad
    for bad in (dict(grad_dtype=2), dict(param_dtype=2), dict(state_dtype=B.BF16)):
        assert call((slot(**bad),)) == 3, bad
    assert call(step_dev=FAKE) == 4 and call(lr_dev=FAKE, ws=FAKE, ws_bytes=8) == 4 and call(lr_dev=FAKE, ws=0x1010, ws_bytes=512) == 1
    assert call(slots=(), n=0) == 0 and call((slot(numel=0, grad=None, param=None),)) == 0


def test_structs_have_the_layout_of_the_header(lib, tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mrl.h"\nint main(void) { printf("%zu %zu %zu %zu %zu\\n",'
                   " sizeof(mrl_norm_params), sizeof(mrl_tensor_slot), sizeof(mrl_adamw_params),"
                   " offsetof(mrl_tensor_slot, weight_decay), offsetof(mrl_adamw_params, lr_dev)); return 0; }\n")
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-I", build.INCLUDE, str(src), "-o", str(exe)], check=True)
    sizes = [int(t) for t in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert sizes == [C.sizeof(B.NormParams), C.sizeof(B.TensorSlotStruct), C.sizeof(B.AdamwParams),
                     B.TensorSlotStruct.weight_decay.offset, B.AdamwParams.lr_dev.offset]
    assert os.path.exists(build.LIB_PATH)


def test_binding_refuses_tensors_it_cannot_describe():
    cpu = torch.zeros(4, 8)
    with pytest.raises(B.MrlError):
        B.TensorSlot(grad=torch.zeros(4, dtype=torch.float16))               # a type without a code
    with pytest.raises(B.MrlError):
        B.TensorSlot(grad=cpu, param=torch.zeros(31))                         # another size
    with pytest.raises(B.MrlError):
        B.TensorSlot(grad=torch.zeros(8, 4).t())                              # not contiguous
    with pytest.raises(B.MrlError):
        B.TensorSlot(grad=cpu, m=torch.zeros(32, dtype=torch.uint8), v=torch.zeros(32))       # two kinds of state
    with pytest.raises(B.MrlError):
        B.mrl_rmsnorm_residual_fwd(cpu, None, torch.ones(8), B.NormParams(1e-6, 0.0, 0, 0), y=cpu.clone())   # host tensors
