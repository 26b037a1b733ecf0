"""What quantizer, product, top tokens and distillation refuse, on the host before a device is touched."""
import ctypes as C

import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

FAKE, OTHER, THIRD = 0x10000, 0x20000, 0x30000       # never dereferenced: every call below fails validation or is a no-op


@pytest.fixture(scope="module")
def lib():
    build.build()
    return B.lib()


def test_quantize_refusals(lib):
    def call(x=FAKE, ld_x=256, dtype=B.BF16, N=4, H=256, rows=128, codes=OTHER, ld_codes=256, scales=THIRD):
        return lib.mrl_e4m3_quantize(x, ld_x, dtype, N, H, rows, codes, ld_codes, scales, None)

    assert call(dtype=B.E4M3) == 3 and call(N=-1) == 1 and call(H=0) == 1
    assert call(rows=0) == 1 and call(rows=64) == 1 and call(rows=-1) == 1
    assert call(ld_x=255) == 1 and call(ld_codes=255) == 1
    assert call(x=None) == 1 and call(codes=None) == 1 and call(scales=None) == 1 and call(codes=FAKE) == 1 and call(codes=THIRD) == 1
    assert call(x=FAKE + 1) == 1 and call(dtype=B.F32, x=FAKE + 2) == 1 and call(scales=THIRD + 2) == 1
    big = (1 << 30) + 1
    assert call(H=big, ld_x=big, ld_codes=big) == 7
    assert call(N=0, x=None) == 0


def test_product_refusals(lib):
    def call(x=FAKE, ld_x=256, xs=0x40000, w=OTHER, ld_w=256, ws=0x50000, N=4, H=256, V=300, dtype=B.BF16, out=THIRD, ld_out=300):
        return lib.mrl_e4m3_product(x, ld_x, xs, w, ld_w, ws, N, H, V, dtype, out, ld_out, None, None)

    assert call(dtype=B.E4M3) == 3 and call(N=-1) == 1 and call(H=0) == 1 and call(V=0) == 1
    assert call(ld_x=240) == 1 and call(ld_w=240) == 1 and call(ld_out=299) == 1
    assert call(ld_x=264) == 1 and call(ld_w=257) == 1 and call(x=FAKE + 8) == 1 and call(w=OTHER + 1) == 1
    assert call(x=None) == 1 and call(xs=None) == 1 and call(w=None) == 1 and call(ws=None) == 1 and call(out=None) == 1
    assert call(xs=0x40002) == 1 and call(out=THIRD + 1) == 1 and call(dtype=B.F32, out=THIRD + 2) == 1 and call(out=FAKE) == 1
    big = (1 << 24) + 16
    assert call(H=big, ld_x=big, ld_w=big) == 7 and call(N=1 << 31) == 7
    assert call(V=(1 << 30) + 1, ld_out=1 << 31) == 7
    assert call(N=0, x=None) == 0


def test_top_refusals(lib):
    def call(z=FAKE, dtype=B.BF16, N=4, V=300, ld=300, ids=OTHER, mask=None, T=1.0, top=5, logp=0x40000, lse=0x50000, ent=None,
             top_ids=0x60000, top_logp=0x70000):
        return lib.mrl_top_logprobs(z, dtype, N, V, ld, ids, mask, T, top, logp, lse, ent, top_ids, top_logp, None, None)

    assert call(dtype=B.E4M3) == 3 and call(N=-1) == 1 and call(V=0) == 1 and call(ld=299) == 1
    for T in (0.0, -1.0, 1e-7, 2e6, float("nan"), float("inf")):
        assert call(T=T) == 1, T
    assert call(top=-1) == 1 and call(top=301) == 1 and call(top=129) == 7 and call(N=1 << 31) == 7
    assert call(top_ids=None) == 1 and call(top_logp=None) == 1 and call(z=None) == 1 and call(ids=None) == 1
    assert call(logp=None, lse=None, top=0) == 1
    assert call(logp=0x50000) == 1 and call(top_logp=0x60000) == 1 and call(lse=FAKE) == 1 and call(top_ids=OTHER) == 1
    assert call(z=FAKE + 1) == 1 and call(dtype=B.F32, z=FAKE + 2) == 1 and call(ids=OTHER + 2) == 1 and call(lse=0x50001) == 1
    assert call(N=0, z=None) == 0


def test_distill_refusals(lib):
    def call(z=FAKE, dtype=B.BF16, N=4, V=300, ld=300, top_ids=OTHER, top_logp=THIRD, top=5, w=None, dp=True, dz=0x40000, ld_out=300,
             kl=None, loss=0x50000, stats=None, ws=0x60000, ws_bytes=1 << 20, **kw):
        base = dict(temperature=1.0, coeff=1.0, direction=0, rest=0, rest_floor=0.0, flags=0, denominator=0.0)
        p = B.DistillParams(**(base | kw))
        return lib.mrl_distill_loss_fwd_bwd(z, dtype, N, V, ld, top_ids, top_logp, top, None, w, p if dp else None, dz, ld_out, kl, loss,
                                            stats, None, ws, ws_bytes, None)

    nan, inf = float("nan"), float("inf")
    assert call(dtype=B.E4M3) == 3 and call(dp=False) == 1 and call(N=-1) == 1 and call(V=0) == 1 and call(ld=299) == 1
    assert call(ld_out=299) == 1 and call(top=0) == 1 and call(top=301) == 1 and call(top=129) == 7
    assert call(V=(1 << 20) + 1, ld=1 << 21, ld_out=1 << 21) == 7 and call(N=1 << 31) == 7
    for bad in (dict(temperature=0.0), dict(temperature=nan), dict(temperature=2e6), dict(coeff=nan), dict(coeff=inf), dict(direction=2),
                dict(direction=-1), dict(rest=2), dict(direction=1, rest=1, rest_floor=0.1), dict(rest_floor=-0.1), dict(rest_floor=1.0),
                dict(rest_floor=nan), dict(direction=1), dict(direction=1, rest_floor=1e-40), dict(flags=2), dict(denominator=inf),
                dict(denominator=nan)):
        assert call(**bad) == 1, bad
    assert call(loss=None) == 1 and call(loss=0x50002) == 1 and call(stats=0x70004) == 1
    assert call(z=None) == 1 and call(top_ids=None) == 1 and call(top_logp=None) == 1
    assert call(z=FAKE + 1) == 1 and call(dz=0x40001) == 1 and call(top_ids=OTHER + 2) == 1 and call(top_logp=THIRD + 1) == 1
    assert call(w=0x70002) == 1 and call(kl=0x70002) == 1 and call(kl=0x50000) == 1
    assert call(dz=FAKE, ld_out=310) == 1                                # in place with another row stride
    assert call(ws=None) == 4 and call(ws_bytes=8) == 4 and call(ws=0x60010) == 1


def test_workspace_sizes(lib):
    a, b = B.workspace_bytes(B.WS_DISTILL, 10, 0), B.workspace_bytes(B.WS_DISTILL, 100000, 0)
    assert 0 < a < b and a % 256 == 0 and b % 256 == 0 and B.workspace_bytes(B.WS_DISTILL, 0, 0) == 0


def test_struct_has_the_layout_of_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "mrl.h"\nint main(void) { printf("%d %d %d %d\\n", '
                   "(int)sizeof(mrl_distill_params), (int)offsetof(mrl_distill_params, rest_floor), "
                   "(int)offsetof(mrl_distill_params, denominator), MRL_MAX_TOP); return 0; }\n")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.run(["gcc", "-I", include, str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(B.DistillParams), B.DistillParams.rest_floor.offset, B.DistillParams.denominator.offset, B.MAX_TOP]


def test_binding_refuses_tensors_that_are_not_on_the_current_device(lib):
    if torch.cuda.is_available():
        pytest.skip("host tensors only")
    z = torch.zeros(2, 8)
    with pytest.raises((B.MrlError, RuntimeError, AssertionError)):
        B.mrl_top_logprobs(z, None, None, 1.0, lse=torch.zeros(2))
