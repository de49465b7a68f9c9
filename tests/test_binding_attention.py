"""The attention side's calls through the binding's compiled part and through Python: the same results in the caller's own
buffers or new ones, the same refusals."""
import sys
import types

import pytest
import torch

import paper_2511_04214_amd as brq

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def test_left_to_python():
    brq.lib()
    n, x, i = brq._native, torch.zeros((2, 4, 64), dtype=BF16), torch.zeros(2, dtype=I32)
    pool = torch.zeros((2, brq.kv4_page_bytes(4, 64)), dtype=torch.uint8)
    assert n.qk_norm_rope(x, None, None, None, 1e-6, None, None, None, False, 1, None, None, None) is None
    assert n.qk_norm_rope_backward(x, None, x, None, None, None, 1e-6, None, None, None, False, 1, None, None, None) is None
    assert n.kv4_append(pool, i.long(), x, x, None, None, None, 1e-6, None, None, None, False, 1, 1, None) is None
    assert n.kv4_read(pool, i.long(), 64, BF16, None, None) is None
    assert n.kv4_attention(x, pool, i.view(2, 1), i, 0.1, True, 0, None, 1, 64, None, None, False, None) is None
    assert n.kv4_pages_copy(pool, i, i) is None and n.kv4_pages_free(i.view(2, 1), i, i, i) is None
    for f in (n.qk_norm_rope, n.qk_norm_rope_backward, n.kv4_append, n.kv4_read, n.kv4_attention, n.kv4_pages_copy, n.kv4_pages_fork, n.kv4_pages_free,
              n.kv4_pages_reserve, n.kv4_pages_compact):
        assert f() is None and f(None) is None
    with pytest.raises(TypeError):
        n.bind_attention(1)
    with pytest.raises(ValueError):
        n.bind_attention(*[0] * 13)


def test_the_library_does_without_a_compiled_part_built_before_these_calls(monkeypatch):
    brq.lib()
    older = types.SimpleNamespace(TORCH=str(torch.__version__), bind=lambda *a: None, bind_stats=lambda *a: None)
    monkeypatch.setattr(brq, "_lib", None)
    monkeypatch.setattr(brq, "_native", None)
    monkeypatch.setattr(brq, "_binding", older, raising=False)
    monkeypatch.setitem(sys.modules, brq.__name__ + "._binding", older)
    with pytest.warns(RuntimeWarning, match="compiled part"):
        brq.lib()
    assert brq._native is None and brq.kv4_page_bytes(2, 64) == 2 * 68 * 64


class Layer:
    """One of every call, on buffers of its own or new ones."""

    def __init__(self, seed=0, T=5, Hq=8, Hk=2, D=64):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.T, self.Hq, self.Hk, self.D = T, Hq, Hk, D
        x = torch.randn((T, Hq + 2 * Hk, D), generator=g, device="cuda").to(BF16)
        self.q, self.k, self.v = x[:, :Hq], x[:, Hq: Hq + Hk], x[:, Hq + Hk:]
        self.gq, self.gk = torch.randn((T, Hq, D), generator=g, device="cuda"), torch.randn((T, Hk, D), generator=g, device="cuda")
        a = torch.rand((40, D // 2), generator=g, device="cuda")
        self.norm = dict(wq=torch.rand(D, generator=g, device="cuda"), wk=torch.rand(D, generator=g, device="cuda"), eps=1e-5, cos=a.cos(), sin=a.sin(),
                         positions=torch.arange(T, device="cuda"), B=32)
        self.first = torch.randint(0, 120, (9, brq.kv4_page_bytes(Hk, D)), generator=g, device="cuda", dtype=torch.uint8)
        self.pool, self.slots = self.first.clone(), torch.arange(T, device="cuda") * 64 + 3
        self.lens = torch.tensor([4, 70, 100], dtype=I32, device="cuda")

    def step(self, **kw):
        q, k = brq.qk_norm_rope(self.q, self.k, **self.norm, **kw)
        out = [q, k, *brq.qk_norm_rope(self.q, None, out_dtype=F32, **kw)[:1], *brq.qk_norm_rope_backward(self.q, self.k, self.gq, self.gk, **self.norm, **kw)]
        out += [brq.kv4_append(self.pool, self.slots, self.k, self.v, q=self.q, Bv=32, **self.norm, **kw), *brq.kv4_read(self.pool, self.slots, self.D, **kw)]
        assert brq.kv4_append(self.pool, self.slots + 1, self.k, self.v, **kw) is None
        table = torch.tensor([[0, -1], [3, 4], [5, 6], [-1, -1], [-1, -1]], dtype=I32, device="cuda")
        lens, refs = torch.cat((self.lens, self.lens[:0].new_zeros(2))), torch.tensor([1, 0, 0, 1, 1, 1, 1, 0, 0], dtype=I32, device="cuda")
        out += [brq.kv4_attention(q[:3], self.pool, table[:3], self.lens, **kw),
                *brq.kv4_attention(q, self.pool, table[1:3], self.lens[1:], 0.2, cu_q=self.lens.new_tensor([0, 3, 5]), max_q=3, want_lse=True, **kw)]
        one = lens.new_tensor
        out += [brq.kv4_pages_fork(self.pool, table, lens, refs, one([1]), one([3]), **kw), brq.kv4_pages_reserve(table, refs, one([0]), one([128]), **kw)]
        brq.kv4_pages_free(table, lens, refs, one([1]), **kw)
        out += [brq.kv4_pages_compact(self.pool, table, refs, **kw), table, lens, refs]
        brq.kv4_pages_copy(self.pool, one([0]), one([8]), **kw)
        return out + [self.pool.clone()]

    def again(self, **kw):
        self.pool.copy_(self.first)
        return self.step(**kw)


def same(a, b):
    return len(a) == len(b) and all((x is None and y is None) or (x.dtype == y.dtype and torch.equal(x, y)) for x, y in zip(a, b))


@pytest.mark.gpu
def test_both_ways_agree(monkeypatch):
    layer = Layer()
    want = layer.again()
    assert same(layer.again(stream=torch.cuda.current_stream()), want)       # (a Stream argument takes the way through Python)
    monkeypatch.setattr(brq, "_native", None)
    assert same(layer.again(), want)


@pytest.mark.gpu
def test_the_caller_s_own_buffers():
    y, T, Hq, Hk, D = Layer(), 5, 8, 2, 64
    want = y.again()
    y.pool.copy_(y.first)
    n = brq._native
    new = lambda H, dt=BF16: torch.zeros((T, H, D), dtype=dt, device="cuda")
    for kw in (dict(), dict(stream=torch.cuda.current_stream())):
        qo, ko = new(Hq), new(Hk)
        r = brq.qk_norm_rope(y.q, y.k, **y.norm, q_out=qo, k_out=ko, **kw)
        assert r[0] is qo and r[1] is ko and torch.equal(qo, want[0]) and torch.equal(ko, want[1])
        dq, dk, ws = new(Hq), new(Hk), torch.zeros(brq.qk_norm_rope_backward_workspace(T, Hq, Hk, D), dtype=torch.uint8, device="cuda")
        r = brq.qk_norm_rope_backward(y.q, y.k, y.gq, y.gk, **y.norm, dq=dq, dk=dk, workspace=ws, **kw)
        assert r[0] is dq and r[1] is dk and same(r, want[3:7])
        qo = new(Hq)
        assert brq.kv4_append(y.pool, y.slots, y.k, y.v, q=y.q, Bv=32, **y.norm, q_out=qo, **kw) is qo and torch.equal(qo, want[7])
        ko, vo = new(Hk), new(Hk)
        r = brq.kv4_read(y.pool, y.slots, D, k_out=ko, v_out=vo, **kw)
        assert r[0] is ko and r[1] is vo and same(r, want[8:10])
    table, lens = torch.tensor([[0, -1], [3, 4], [5, 6]], dtype=I32, device="cuda"), y.lens
    brq.kv4_append(y.pool, y.slots + 1, y.k, y.v)
    out, lse = torch.zeros((3, Hq, D), dtype=BF16, device="cuda"), torch.zeros((3, Hq), device="cuda")
    for kw in (dict(), dict(stream=torch.cuda.current_stream())):
        assert brq.kv4_attention(want[0][:3], y.pool, table, lens, out=out, **kw) is out and torch.equal(out, want[10])
        r = brq.kv4_attention(want[0][:3], y.pool, table, lens, out=out, lse=lse, **kw)
        assert r[0] is out and r[1] is lse and bool((lse != 0).all())
    with pytest.raises(brq.BrqError) as e:
        big = torch.zeros((1, 4000), dtype=I32, device="cuda")
        brq.kv4_attention(want[0][:1], y.pool, big, lens[:1], workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 2
    assert n.kv4_attention(want[0][:3].as_subclass(type("Named", (torch.Tensor,), {})), y.pool, table, lens, 0.1, True, 0, None, 1, 64, None, None, False, None) is None


@pytest.mark.gpu
def test_calls_go_to_the_current_stream():
    layer, side = Layer(1), torch.cuda.Stream()
    want = [None if t is None else t.cpu() for t in layer.again()]
    torch.cuda.synchronize()
    a = torch.randn((8192, 8192), device="cuda")
    out = torch.empty_like(a)
    with torch.cuda.stream(side):
        layer.again()
        torch.cuda.current_stream().synchronize()
    for _ in range(30):
        torch.mm(a, a, out=out)
    late = torch.cuda.current_stream().record_event()
    with torch.cuda.stream(side):
        got = [None if t is None else t.cpu() for t in layer.again()]
    assert not late.query(), "the default stream was not busy long enough: this shows nothing"
    assert same(got, want)
    torch.cuda.synchronize()
