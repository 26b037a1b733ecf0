"""Tensors of an update that are one another are refused on the host: two would be written through one address."""
import itertools

import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build


@pytest.mark.parametrize("pair", list(itertools.combinations(("grad", "param", "master", "m", "v"), 2)))
def test_one_buffer_for_two_of_a_tensor_is_refused(pair):
    build.build()
    at = dict(grad=0x1000, param=0x2000, master=0x3000, m=0x4000, v=0x5000)      # never dereferenced: the call fails validation
    at[pair[1]] = at[pair[0]]
    good = B.TensorSlotStruct(**dict(grad=None, param=None, m=None, v=None, numel=0))
    bad = B.TensorSlotStruct(**at, numel=64, grad_dtype=B.BF16, param_dtype=B.BF16, state_dtype=B.F32)
    ap = B.AdamwParams(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    assert B.lib().mrl_adamw_step((B.TensorSlotStruct * 2)(good, bad), 2, ap, None, None, None, 0, None) == 1


def test_one_scale_array_for_both_states_is_refused():
    build.build()
    bad = B.TensorSlotStruct(grad=0x1000, param=0x2000, m=0x4000, v=0x5000, m_scale=0x6000, v_scale=0x6000, numel=64, state_dtype=B.E4M3)
    ap = B.AdamwParams(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    assert B.lib().mrl_adamw_step((B.TensorSlotStruct * 1)(bad), 1, ap, None, None, None, 0, None) == 1
