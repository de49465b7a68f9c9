"""Attention's scale is a number: NaN and infinities are refused."""
import ctypes
import math
from ctypes import byref

import pytest
import torch

import paper_2511_04214_amd as brq
from paper_2511_04214_amd.attention import _Heads

SHAPE = 2
P = 0x1000          # never dereferenced


@pytest.mark.parametrize("scale", [math.nan, math.inf, -math.inf])
def test_a_scale_that_is_no_number_is_refused(scale):
    h = byref(_Heads(P, 8, 8 * 64, 64))
    for T in (0, 6):
        assert brq.lib().brq_kv4_attention(h, T, 64, P, 9, 2, P, 4, P, P, 3, scale, 1, 0, 4, 256, h, None, P, ctypes.c_int64(1 << 40), None) == SHAPE


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [math.nan, math.inf])
def test_the_binding_refuses_it(scale):
    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    pool, i = torch.zeros((2, brq.kv4_page_bytes(4, 64)), dtype=torch.uint8, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(brq.BrqError):
        brq.kv4_attention(x, pool, i[:, None].contiguous(), i, scale)
