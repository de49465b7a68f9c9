"""Pages of the cache on the device against a scheduler in plain Python, one pair after the other."""
import random

import pytest
import torch

import paper_2511_04214_amd as brq

pytestmark = pytest.mark.gpu
I32 = torch.int32


class State:
    """refs, table, lens, pool as lists; what a call does to them, in order."""

    def __init__(self, r, pages, seqs, cols, page_bytes, lens, slack=0):
        self.cols, self.pages = cols, pages
        self.pool = torch.randint(0, 256, (pages, page_bytes), dtype=torch.uint8)
        self.refs, self.table, self.lens = [0] * pages, [[-1] * cols for _ in range(seqs)], list(lens) + [0] * (seqs - len(lens))
        free = r.sample(range(pages), pages)
        for s, n in enumerate(lens):
            for c in range(min(cols, -(-n // 64) + (r.randint(0, slack) if n else 0))):
                self.table[s][c] = free.pop()
                self.refs[self.table[s][c]] = 1

    def device(self):
        self.d = [self.pool.clone().cuda(), torch.tensor(self.table, dtype=I32).cuda(), torch.tensor(self.lens, dtype=I32).cuda(), torch.tensor(self.refs, dtype=I32).cuda()]
        return self.d

    def same(self):
        pool, table, lens, refs = self.d
        return (table.tolist() == self.table and lens.tolist() == self.lens and refs.tolist() == self.refs and torch.equal(pool.cpu(), self.pool))

    def fork(self, parents, children):
        S = len(self.table)
        free = [p for p in range(self.pages) if self.refs[p] == 0]
        old = [list(row) for row in self.table]
        failed = 0
        for p, c in zip(parents, children):
            if not (0 <= p < S and 0 <= c < S):
                continue
            n, row = self.lens[p], [-1] * self.cols
            if n % 64:
                if not free:
                    failed += 1
                    self.table[c], self.lens[c] = row, 0
                    continue
                row[n // 64] = free.pop(0)
                self.refs[row[n // 64]] = 1
                self.pool[row[n // 64]] = self.pool[old[p][n // 64]]
            for k in range(n // 64):
                row[k] = old[p][k]
                self.refs[row[k]] += 1
            self.table[c], self.lens[c] = row, n
        return failed

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.table):
                for e in self.table[s]:
                    if e >= 0:
                        self.refs[e] -= 1
                self.table[s], self.lens[s] = [-1] * self.cols, 0

    def reserve(self, seqs, tokens):
        free = [p for p in range(self.pages) if self.refs[p] == 0]
        asked = failed = 0
        for s, n in zip(seqs, tokens):
            if not 0 <= s < len(self.table) or n <= 0:
                continue
            cols = -(-n // 64)
            if cols > self.cols:
                failed += 1
                continue
            empty = [c for c in range(cols) if self.table[s][c] < 0]
            if empty and asked + len(empty) > len(free):
                failed += 1
            else:
                for i, c in enumerate(empty):
                    self.table[s][c] = free[asked + i]
                    self.refs[free[asked + i]] = 1
            asked += len(empty)
        return failed

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        high = [p for p in range(live, self.pages) if self.refs[p] > 0]
        to = dict(zip(high, holes))
        for a, b in to.items():
            self.pool[b], self.refs[b], self.refs[a] = self.pool[a], self.refs[a], 0
        self.table = [[to.get(e, e) for e in row] for row in self.table]
        return live


def ints(x):
    return torch.tensor(list(x), dtype=I32, device="cuda")


@pytest.mark.parametrize("pages,seqs,cols,page_bytes,seed", [(40, 6, 5, 16, 0), (3000, 50, 20, 4352, 1), (20000, 40, 70, 32, 2), (33, 8, 3, 8704 * 3, 3), (200, 70, 4, 16400, 4), (40000, 400, 90, 16, 5)])
def test_a_scheduler_s_day(pages, seqs, cols, page_bytes, seed):
    r = random.Random(seed)
    half = seqs // 2
    lens = [r.choice([0, 1, 63, 64, 65, 128, r.randint(0, cols * 64)]) for _ in range(half)]
    while sum(-(-n // 64) for n in lens) > pages * 0.6:
        lens = [n // 2 for n in lens]
    st = State(r, pages, seqs, cols, page_bytes, lens)
    pool, table, lens_d, refs = st.device()
    parents, children = [r.randrange(half) for _ in range(half)], r.sample(range(half, seqs), half)
    f = brq.kv4_pages_fork(pool, table, lens_d, refs, ints(parents), ints(children))
    assert f.tolist() == [st.fork(parents, children)] and st.same()
    gone = r.sample(range(seqs), seqs // 3)
    brq.kv4_pages_free(table, lens_d, refs, ints(gone))
    st.free(gone)
    assert st.same()
    who = r.sample(range(seqs), seqs // 2)
    tokens = [r.choice([0, -3, 1, 64, 65, cols * 64, cols * 64 + 1, r.randint(0, cols * 64)]) for _ in who]
    f = brq.kv4_pages_reserve(table, refs, ints(who), ints(tokens))
    assert f.tolist() == [st.reserve(who, tokens)] and st.same()
    live = brq.kv4_pages_compact(pool, table, refs)
    assert live.tolist() == [st.compact()] and st.same()
    assert brq.kv4_pages_compact(pool, table, refs).tolist() == [st.compact()] and st.same()        # dense already


def test_no_page_left():
    r = random.Random(7)
    st = State(r, 10, 12, 4, 64, [100, 100, 64, 1, 30], 0)          # 7 pages taken
    pool, table, lens, refs = st.device()
    pairs = ([0, 1, 2, 3, 4, 0], [6, 7, 8, 9, 10, 11])               # 5 want one, 3 are left
    assert brq.kv4_pages_fork(pool, table, lens, refs, ints(pairs[0]), ints(pairs[1])).tolist() == [st.fork(*pairs)] == [2]
    assert st.same()
    assert brq.kv4_pages_reserve(table, refs, ints([0, 5]), ints([200, 1])).tolist() == [st.reserve([0, 5], [200, 1])] == [2]
    assert st.same()
    brq.kv4_pages_free(table, lens, refs, ints([6, 7]))
    st.free([6, 7])
    assert brq.kv4_pages_reserve(table, refs, ints([5, 0, 6, 7]), ints([64, 999, 256, 64])).tolist() == [st.reserve([5, 0, 6, 7], [64, 999, 256, 64])]
    assert st.same()


def test_lists_with_numbers_that_are_none_and_nothing_to_do():
    st = State(random.Random(8), 12, 5, 3, 32, [70, 64, 0])
    pool, table, lens, refs = st.device()
    none = [-1, 5, 1 << 30, -(1 << 31)]
    assert brq.kv4_pages_fork(pool, table, lens, refs, ints(none + [0]), ints([3] * 4 + [99])).tolist() == [0]
    assert brq.kv4_pages_fork(pool, table, lens, refs, ints([0, 2]), ints([-7, 4])).tolist() == [st.fork([2], [4])]
    brq.kv4_pages_free(table, lens, refs, ints(none))
    assert brq.kv4_pages_reserve(table, refs, ints(none), ints([64] * 4)).tolist() == [0]
    brq.kv4_pages_copy(pool, ints([0, -1, 12, 3, 3]), ints([12, 0, 1, 3, -1]))
    empty = ints([])
    assert brq.kv4_pages_fork(pool, table, lens, refs, empty, empty).tolist() == [0]
    assert brq.kv4_pages_reserve(table, refs, empty, empty).tolist() == [0]
    brq.kv4_pages_free(table, lens, refs, empty)
    brq.kv4_pages_copy(pool, empty, empty)
    assert st.same()
    brq.kv4_pages_free(table, lens, refs, ints([0, 0, 0]))           # named three times, given up once
    st.free([0])
    assert st.same()
    dangling = table.clone()
    dangling[1, 2] = 11                                              # an entry that names a page nobody holds
    live = brq.kv4_pages_compact(pool, dangling, refs)
    st.compact()
    assert dangling.tolist()[1][2] == -1 and torch.equal(refs.cpu(), torch.tensor(st.refs, dtype=I32)) and live.tolist() == [1]


def test_copy():
    pool = torch.randint(0, 256, (50, 8704), dtype=torch.uint8)
    d = pool.cuda()
    src, dst = random.Random(9).sample(range(25), 20), random.Random(10).sample(range(25, 50), 20)
    brq.kv4_pages_copy(d, ints(src), ints(dst))
    pool[dst] = pool[src]
    assert torch.equal(d.cpu(), pool)


def test_a_forked_sequence_goes_its_own_way():
    """Parent and child share a prefix, write different tokens behind it, and read their own; dense or not."""
    g = torch.Generator().manual_seed(1)
    Hk, D, n = 2, 64, 70
    pool = torch.zeros((9, brq.kv4_page_bytes(Hk, D)), dtype=torch.uint8, device="cuda")
    table, lens, refs = torch.full((2, 3), -1, dtype=I32, device="cuda"), ints([0, 0]), torch.zeros(9, dtype=I32, device="cuda")
    refs[0], refs[3] = 1, 1                                          # somebody else's
    brq.kv4_pages_reserve(table, refs, ints([0]), ints([n]))
    x = torch.randn((n + 2, Hk, D), generator=g).to(torch.bfloat16).cuda()

    def put(s, tokens, at):
        at = torch.as_tensor(at, device="cuda")
        brq.kv4_append(pool, table[s].long()[at // 64] * 64 + at % 64, tokens, tokens)
    put(0, x[:n], torch.arange(n))
    lens[0] = n
    brq.kv4_pages_fork(pool, table, lens, refs, ints([0]), ints([1]))
    assert table.tolist() == [[1, 2, -1], [1, 4, -1]] and refs.tolist() == [1, 2, 1, 1, 1, 0, 0, 0, 0]
    put(0, x[n: n + 1], [n])
    put(1, x[n + 1:], [n])
    lens += 1
    q = torch.randn((2, 4, D), generator=g).to(torch.bfloat16).cuda()
    out = brq.kv4_attention(q, pool, table, lens)
    assert not torch.equal(out[0], out[1])
    alone = torch.zeros((2, brq.kv4_page_bytes(Hk, D)), dtype=torch.uint8, device="cuda")
    for s, last in ((0, n), (1, n + 1)):
        t = torch.tensor([[0, 1]], dtype=I32, device="cuda")
        brq.kv4_append(alone, torch.arange(n + 1, device="cuda"), torch.cat((x[:n], x[last: last + 1])), torch.cat((x[:n], x[last: last + 1])))
        assert torch.equal(brq.kv4_attention(q[s: s + 1], alone, t, lens[s: s + 1], max_kv=192), out[s: s + 1])
    refs[0], refs[3] = 0, 0
    assert brq.kv4_pages_compact(pool, table, refs).tolist() == [3]
    assert torch.equal(brq.kv4_attention(q, pool, table, lens), out)


def test_in_a_graph():
    st = State(random.Random(11), 60, 10, 4, 4352, [100, 64, 130, 20, 10])
    start = [x.clone() for x in st.device()]
    pool, table, lens, refs = st.d
    lists = [ints([0, 1, 2]), ints([5, 6, 7]), ints([0, 3]), ints([5, 6]), ints([200, 100])]
    graph = torch.cuda.CUDAGraph()

    def day():
        return (brq.kv4_pages_fork(pool, table, lens, refs, lists[0], lists[1]), brq.kv4_pages_free(table, lens, refs, lists[2]),
                brq.kv4_pages_reserve(table, refs, lists[3], lists[4]), brq.kv4_pages_compact(pool, table, refs))
    with torch.cuda.graph(graph):
        r = day()
    st.fork([0, 1, 2], [5, 6, 7]), st.free([0, 3]), st.reserve([5, 6], [200, 100])
    live = st.compact()
    for _ in range(3):
        for x, y in zip(st.d, start):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert st.same() and r[3].tolist() == [live]
