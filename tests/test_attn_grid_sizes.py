"""Sizes that one grid of the attention kernels could not hold are refused on the host."""
import ctypes

import pytest

import paper_2511_04214_amd as brq

OK = 0


def workspace(T, S, Hq, Hk, D=64, max_q=1, max_kv=64):
    n = ctypes.c_int64(-1)
    return brq.lib().brq_kv4_attention_workspace(T, S, Hq, Hk, D, max_q, max_kv, ctypes.byref(n)), n.value


@pytest.mark.parametrize("S,Hq,Hk", [(1 << 22, 1, 1), (1 << 19, 8, 8), (1 << 16, 64, 64), (1 << 20, 16, 4)])
def test_too_many_sequences(S, Hq, Hk):
    shape = workspace(1, 1, 1, 1, D=96)[0]               # no such head: a refused shape
    assert shape != OK
    assert workspace(0, S, Hq, Hk) == (shape, -1)
    assert workspace(0, S - 1, Hq, Hk) == (OK, 0)
