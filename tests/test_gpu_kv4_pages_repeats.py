"""Reservations that name a row again and again: no count passes what holds it, and no page is taken that there is not."""
import pytest
import torch

import paper_2511_04214_amd as brq

pytestmark = pytest.mark.gpu
I32 = torch.int32


@pytest.mark.parametrize("n,cols", [(1024, 1 << 21), (2048, 1 << 21), (1100, (1 << 21) + 5), (65, 1 << 22), (64, 1 << 24)])
def test_wants_past_32_bits(n, cols):
    """n times `cols` columns of one row: 2^31 and more within a count of 1024 rows, then a few; far more than there are pages."""
    table = torch.full((1, cols), -1, dtype=I32, device="cuda")
    refs = torch.tensor([0, 1, 0, 0, 1, 0, 0, 0], dtype=I32, device="cuda")
    before = refs.clone()
    seqs, tokens = torch.zeros(n, dtype=I32, device="cuda"), torch.full((n,), min(cols * 64, (1 << 31) - 1), dtype=I32, device="cuda")
    assert int(brq.kv4_pages_reserve(table, refs, seqs, tokens)) == n
    assert int((table != -1).sum()) == 0 and torch.equal(refs, before)


def test_rows_named_twice_among_others():
    """What is in the table afterwards are free pages, no page twice; rows of their own get what they ask for."""
    g = torch.Generator().manual_seed(81)
    for n in (40, 300):
        table, refs = torch.full((n, 6), -1, dtype=I32, device="cuda"), torch.zeros(4000, dtype=I32, device="cuda")
        seqs = torch.arange(n, dtype=I32)
        seqs[1::2] = seqs[::2]
        tokens = torch.randint(1, 385, (n,), generator=g).to(I32)
        brq.kv4_pages_reserve(table, refs, seqs.cuda(), tokens.cuda())
        t, r = table.cpu(), refs.cpu()
        pages = t[t >= 0]
        assert len(pages.unique()) == len(pages) and int(pages.max()) < 4000 and bool((r[pages.long()] == 1).all())
        for s in range(0, n, 2):
            need = -(-int(tokens[s: s + 2].max()) // 64)
            assert (t[s, :need] >= 0).all() and (t[s, need:] == -1).all() and (t[s + 1] == -1).all()


def test_children_that_are_parents():
    """A pair's child as another's parent in one call: whose state is copied is not said, but pages stay pages."""
    for cols in (1, 3):
        S, n = 300, 40
        table, refs = torch.full((S, cols), -1, dtype=I32, device="cuda"), torch.zeros(2000, dtype=I32, device="cuda")
        lens = torch.zeros(S, dtype=I32, device="cuda")
        first = torch.arange(n, dtype=I32, device="cuda")
        assert int(brq.kv4_pages_reserve(table, refs, first, torch.full((n,), cols * 64, dtype=I32, device="cuda"))) == 0
        lens[:n:2], lens[1:n:2] = cols * 64, cols * 64 - 7
        pool = torch.zeros((2000, 4352), dtype=torch.uint8, device="cuda")
        brq.kv4_pages_fork(pool, table, lens, refs, torch.arange(250, dtype=I32, device="cuda"), torch.arange(n, n + 250, dtype=I32, device="cuda"))
        t = table.cpu()
        assert bool(((t >= -1) & (t < 2000)).all()) and bool((lens.cpu() <= cols * 64).all()) and bool((refs.cpu() >= 0).all())
