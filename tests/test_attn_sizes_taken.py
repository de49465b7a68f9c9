"""Bounds on the longest sequence do not multiply with the number of sequences: a call of few rows is taken whatever max_q says."""
import ctypes

import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq
import test_gpu_kv4_attention as base

OK, SHAPE = 0, 2


def sizes(S, Hq, Hk, max_q, T=0, D=64):
    n = ctypes.c_int64(-1)
    return brq.lib().brq_kv4_attention_workspace(T, S, Hq, Hk, D, max_q, 1000, ctypes.byref(n))


@pytest.mark.parametrize("S,Hq,Hk,max_q", [(1024, 32, 8, 65536), (1 << 17, 32, 8, 1 << 20), ((1 << 22) - 1, 64, 1, (1 << 25) - 1), (1, 64, 1, (1 << 25) - 1), (64, 65535, 1, 1 << 15)])
def test_taken(S, Hq, Hk, max_q):
    assert sizes(S, Hq, Hk, max_q) == OK


@pytest.mark.parametrize("S,Hq,Hk,max_q,T", [(1 << 22, 1, 1, 1, 0), (1, 1, 1, 1 << 25, 0), (1, 1, 1, 0, 0), (1, 65536, 1, 1, 0), (1, 32, 8, 1, 1 << 20)])
def test_the_limits_that_are_left(S, Hq, Hk, max_q, T):
    assert sizes(S, Hq, Hk, max_q, T) == SHAPE


@pytest.mark.gpu
def test_a_batch_of_many_short_sequences():
    """8192 sequences of 2 rows without a bound: as with it, and as the formulas have it."""
    g = torch.Generator().manual_seed(91)
    S, Hq, Hk, D = 8192, 16, 2, 64
    pool = base.cache(g, 50, Hk, D)
    table = torch.randint(0, 50, (S, 3), generator=g).to(torch.int32)
    lens = torch.randint(0, 193, (S,), generator=g).to(torch.int32)
    q = torch.randn((2 * S, Hq, D), generator=g).to(torch.bfloat16)
    cu = torch.arange(0, 2 * S + 1, 2, dtype=torch.int32)
    some = torch.randperm(S, generator=g)[:40].tolist() + [0, S - 1]
    rows = torch.tensor([r for s in some for r in (2 * s, 2 * s + 1)])
    want = ref.attention(q[rows], ref.cache_values(pool, Hk, D), table[some], lens[some].tolist(), D ** -0.5, True, 0, torch.arange(0, 2 * len(some) + 1, 2), 2, 192)
    for max_q in (None, 2 * S, 2):
        out, lse = brq.kv4_attention(q.cuda(), pool.cuda(), table.cuda(), lens.cuda(), cu_q=cu.cuda(), max_q=max_q, want_lse=True)
        base.check(out[rows.cuda()], want, lse[rows.cuda()])
