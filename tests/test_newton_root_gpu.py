"""The square root of the 8-bit second moment (newton_root) against the IEEE root, for every float of the range it is used on."""
import ctypes as C
import shutil
import subprocess

import pytest
import torch

from paper_2605_07244_b200 import build

pytestmark = pytest.mark.gpu

SOURCE = r"""
#include "mrl_common.cuh"
// every float from `lo` to `hi` (as ordered bits), in both places of a pair: how many differ from the IEEE root, how many there were
__global__ void compare(uint32_t lo, uint32_t hi, unsigned long long* out) {
  unsigned long long bad = 0, seen = 0;
  for (uint64_t b = (uint64_t)lo + blockIdx.x * blockDim.x + threadIdx.x; b <= hi; b += (uint64_t)gridDim.x * blockDim.x) {
    const float v = __uint_as_float((uint32_t)b), other = __uint_as_float(lo + hi - (uint32_t)b);
    const float2 r = mrl::split_f2(mrl::newton_root(mrl::make_f2(v, other)));
    bad += (__float_as_uint(r.x) != __float_as_uint(__fsqrt_rn(v))) + (__float_as_uint(r.y) != __float_as_uint(__fsqrt_rn(other)));
    ++seen;
  }
  atomicAdd(out, bad);
  atomicAdd(out + 1, seen);
}
extern "C" int run(void* out) {
  const float lo = mrl::kRootMin, hi = mrl::kRootMax;
  uint32_t l, h;
  memcpy(&l, &lo, 4), memcpy(&h, &hi, 4);
  compare<<<1184, 256>>>(l, h, static_cast<unsigned long long*>(out));
  return (int)cudaGetLastError();
}
"""


def test_every_float_of_the_range_has_the_ieee_root(tmp_path):
    if shutil.which("nvcc") is None:
        pytest.skip("no nvcc")
    (tmp_path / "root.cu").write_text("#include <string.h>\n" + SOURCE)
    so = tmp_path / "root.so"
    subprocess.run(["nvcc", *build.NVCC_FLAGS, "-I", build.INCLUDE, "-I", build.CSRC, "-o", str(so), str(tmp_path / "root.cu")], check=True)
    out = torch.zeros(2, dtype=torch.int64, device="cuda")
    assert C.CDLL(str(so)).run(C.c_void_p(out.data_ptr())) == 0
    torch.cuda.synchronize()
    bits = [int(torch.tensor(v, dtype=torch.float32).view(torch.int32)) for v in (1e-25, 1e37)]
    assert out.tolist() == [0, bits[1] - bits[0] + 1]
