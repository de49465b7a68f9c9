"""Which kernel attention takes for a call, on the CPU (host arithmetic for a device of 256 compute units).  The tests of
test_gpu_kv4_attention_routes.py say of each call that it runs the kernel that it is about."""
import ctypes
import random

import pytest

import paper_2511_04214_amd as brq
from kv4_forms import FORMS, GROUPED, NAN, plan

ROUTE = brq.diag_kv4_attention_route


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_the_forms_of_the_gpu_tests(form, D):
    """Every kernel for many rows is among them, with every mask."""
    for causal, window in ((True, 0), (True, 1), (True, 70), (True, 500), (False, 0)):
        got = plan(form, D, FORMS, 527, 290, causal, window)
        if D == 64:
            assert got[0] == ("one" if form == "one" else "pair")
        else:
            assert got[0] == form.split()[0]
        assert (got[1] > 1) == (form == "pair in parts" and window in (0, 500))


@pytest.mark.parametrize("form", FORMS)
def test_the_other_forms(form):
    S, Hk, max_kv = GROUPED[form]
    assert ROUTE(527, S, 3 * Hk, Hk, 128, 290, max_kv)[0] == form.split()[0]
    S, Hk, max_kv, q = NAN[form]
    got = ROUTE(S * q, S, Hk, Hk, 128, q, max_kv, causal=False)
    assert got[0] == form.split()[0] and (got[1] > 1) == ("parts" in form)


@pytest.mark.parametrize("D", [64, 128])
def test_up_to_32_rows(D):
    for q, G, want in ((1, 1, "few_16"), (1, 16, "few_16"), (16, 1, "few_16"), (4, 4, "few_16"), (1, 17, "few_32"), (17, 1, "few_32"), (4, 8, "few_32"), (32, 1, "few_32"),
                       (33, 1, "one"), (3, 11, "one"), (1, 33, "one")):
        assert ROUTE(q * 8, 8, 2 * G, 2, D, q, 300)[0] == want


def test_prompts():
    for n, want in ((64, "one"), (384, "one"), (385, "pair"), (1024, "pair"), (2048, "pair"), (3000, "tall"), (8192, "tall"), (100000, "tall")):
        assert ROUTE(n, 1, 32, 8, 128, n, n)[0] == want
        assert ROUTE(n, 1, 16, 4, 64, n, n)[0] == ("one" if want == "one" else "pair")


def test_parts():
    """Of contexts of more than 16 pages for few rows, of more than 8 for many, where the tiles leave units idle."""
    for pages, want in ((1, 1), (16, 1), (17, 3), (64, 8), (2048, 256)):
        assert ROUTE(1, 1, 4, 1, 128, 1, pages * 64)[1] == want
    for pages, want in ((7, 1), (8, 1), (9, 3), (16, 4)):
        assert ROUTE(64, 1, 4, 2, 128, 64, pages * 64) == ("pair", want)
    assert ROUTE(1, 1, 32, 8, 128, 1, 131072) == ("few_16", 32) and ROUTE(64, 64, 32, 8, 128, 1, 2000)[1] == 1 and ROUTE(64, 64, 32, 8, 128, 1, 8192)[1] > 1


def test_a_mask_never_asks_for_more_parts_than_the_workspace_has():
    """The workspace is sized without causality and window."""
    r = random.Random(7)
    for _ in range(20000):
        S, Hk = int(2 ** r.uniform(0, 9)), int(2 ** r.uniform(0, 6))
        max_q, G = int(2 ** r.uniform(0, 13)), int(2 ** r.uniform(0, 5))
        T = min(S * max_q, ((1 << 25) - 1) // (Hk * G))
        a = (T, S, Hk * G, Hk, r.choice((64, 128)), max_q, int(2 ** r.uniform(0, 18)))
        most = ROUTE(*a, causal=False)[1]
        assert ROUTE(*a)[1] <= most and ROUTE(*a, window=int(2 ** r.uniform(0, 18)))[1] <= most, a


def test_refusals():
    n = ctypes.c_int32()
    call = brq.lib().brq_diag_kv4_attention_route
    good = (6, 3, 8, 2, 64, 4, 256, 1, 0, 256)
    assert call(*good, ctypes.byref(n), ctypes.byref(n)) == 0
    assert call(*good, None, ctypes.byref(n)) == call(*good, ctypes.byref(n), None) == 1
    for i, bad in ((0, 0), (0, -1), (0, 1 << 31), (0, 1 << 23), (1, 0), (2, 7), (3, 0), (4, 96), (5, 0), (6, -1), (8, -1), (8, 1 << 31), (9, 0), (9, 1 << 31)):
        assert call(*good[:i], bad, *good[i + 1:], ctypes.byref(n), ctypes.byref(n)) == 2
    assert call(*good[:7], 0, 5, 256, ctypes.byref(n), ctypes.byref(n)) == 2                # a window without causality
