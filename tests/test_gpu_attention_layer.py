"""The example of an attention layer: what its calls get and give, against 64 bits, and what page moves must not change."""
import math
import os
import sys

import pytest
import torch

import attn_ref as ref
import paper_2511_04214_amd as brq

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import attention_layer as ex  # noqa: E402

pytestmark = pytest.mark.gpu


def ids(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


def made(Hq, Hk, D, C=256, tokens=512, B=32):
    g = torch.Generator().manual_seed(Hq * D)
    w = lambda *s: torch.randn(s, generator=g).div(s[-1] ** 0.5).bfloat16().cuda()                         # noqa: E731
    norms = [(1 + 0.1 * torch.randn(D, generator=g)).cuda() for _ in range(2)]
    return ex.Attention(w((Hq + 2 * Hk) * D, C), w(C, Hq * D), *norms, Hq, Hk, D, tokens, B), g


@pytest.mark.parametrize("Hq,Hk,D,B", [(4, 2, 64, 32), (8, 2, 128, 32), (3, 1, 128, 128)])
def test_layer(Hq, Hk, D, B, monkeypatch):
    layer, g = made(Hq, Hk, D, B=B)
    seen = []
    append, attend = brq.kv4_append, brq.kv4_attention
    monkeypatch.setattr(brq, "kv4_append", lambda *a, **k: seen.append((a, k, append(*a, **k))) or seen[-1][2])
    monkeypatch.setattr(brq, "kv4_attention", lambda *a, **k: seen.append((a, k, attend(*a, **k))) or seen[-1][2])
    cache = ex.Cache(20, 3, 512, Hk, D)
    for tokens in ((70, 1, 130), (1, 1, 1), (5, 64, 2)):
        del seen[:]
        x = torch.randn((sum(tokens), 256), generator=g).bfloat16().cuda()
        before = [int(n) for n in cache.lens]
        y = layer(x, cache, ids(0, 1, 2), ids(*tokens), max(tokens), 512)
        (pool, slots, k, v, q), kw, q2 = seen[0][0][:5], seen[0][1], seen[0][2]
        # positions and slots: every token's own
        want = torch.cat([torch.arange(b, b + n) for b, n in zip(before, tokens)])
        assert torch.equal(kw["positions"].cpu(), want)
        assert len(set(slots.tolist())) == len(slots)
        # queries: rounded once to bfloat16, 32-bit arithmetic before
        f, m = ref.forward(q.cpu(), layer.wq.cpu(), 1e-6, layer.cos.cpu(), layer.sin.cpu(), want, False, B)
        assert ((q2.cpu().double() - f).abs() <= 2.0 ** -8 * f.abs() + 2.0 ** -18 * m).all()
        # what stands in the cache: keys and values within half a step of the codes' grid, 1 of a block's largest over 4 to 6
        got = brq.kv4_read(cache.pool, slots, D, torch.float32)
        kf = ref.forward(k.cpu(), layer.wk.cpu(), 1e-6, layer.cos.cpu(), layer.sin.cpu(), want, False, B)[0]
        for a, b in ((got[0], kf), (got[1], ref.rotate(v.cpu().double(), B))):
            top = b.reshape(*b.shape[:-1], -1, 32).abs().amax(-1).repeat_interleave(32, -1)
            assert ((a.cpu().double() - b).abs() <= top * (1 / 4 + 2.0 ** -16)).all()
        # attention over the cache as it stands
        o = seen[1][2]
        lens = [b + n for b, n in zip(before, tokens)]
        cu = torch.tensor([0, *tokens]).cumsum(0)
        out, _, mag, ds = ref.attention(q2.cpu(), ref.cache_values(cache.pool.cpu(), Hk, D), cache.table.cpu(), lens, D ** -0.5, True, 0, cu, max(tokens), 512)
        bound = 2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * ds[..., None] + 2.0 ** -18) * mag + 1e-30
        assert ((o.cpu().double() - out).abs() <= bound).all()
        # the output projection: products of codes exact, sums of Hq D of them in 32 bits, rounded once
        a = ref.code_values(*(t.cpu() for t in brq.mxfp4_quantize(o.view(len(x), -1))))
        w = ref.code_values(*(t.cpu() for t in layer.o))
        e = (y.cpu().double() - a @ w.T).abs()
        assert (e <= 2.0 ** -8 * (a @ w.T).abs() + 1e-5 * (a.abs() @ w.abs().T)).all()


def test_values_come_out_in_the_rotated_basis():
    """One token, one head: the output is its value as it stands in the cache, rotated; turned back it is the value again up to the
    quantizer.  32 equal magnitudes just below 1 are 8 steps of their block's scale, of which the codes have 6."""
    D, B = 64, 32
    v = torch.zeros((1, 1, D), dtype=torch.bfloat16)
    v[0, 0, 5] = 2.0 ** 0.5 * 4
    v = v.cuda()
    pool = torch.zeros((1, brq.kv4_page_bytes(1, D)), dtype=torch.uint8, device="cuda")
    brq.kv4_append(pool, torch.zeros(1, dtype=torch.int64, device="cuda"), v, v, Bv=B)
    o = brq.kv4_attention(v, pool, ids(0).view(1, 1), ids(1))
    back = brq.block_rotate(o.view(1, D), B, out_dtype=torch.float32).cpu()          # H H / B = 1
    want = torch.zeros(1, D)
    want[0, 5] = 0.75 * 2.0 ** 0.5 * 4
    assert torch.allclose(back, want, atol=2.0 ** -6)


def test_forks_and_moved_pages_change_nothing():
    """A fork goes on as its parent does, bit for bit, and so does a sequence whose pages were moved."""
    layer, g = made(8, 2, 128)
    a, b = ex.Cache(30, 4, 512, 2, 128), ex.Cache(30, 4, 512, 2, 128)
    x = torch.randn((290, 256), generator=g).bfloat16().cuda()
    for c in (a, b):
        assert torch.equal(layer(x, c, ids(0, 1, 2), ids(150, 100, 40), 150, 512), layer(x, ex.Cache(30, 4, 512, 2, 128), ids(0, 1, 2), ids(150, 100, 40), 150, 512))
        c.fork(ids(1), ids(3))
    for _ in range(3):
        x = torch.randn((3, 256), generator=g).bfloat16().cuda()[[0, 1, 2, 1]].contiguous()
        ya, yb = (layer(x, c, ids(0, 1, 2, 3), ids(1, 1, 1, 1), 1, 512) for c in (a, b))
        assert torch.equal(ya, yb) and torch.equal(ya[1], ya[3])
    for c in (a, b):
        c.free(ids(0, 1))
    pages = a.table[2:][a.table[2:] >= 0].unique().numel()
    assert a.compact() == pages and int((a.refs > 0).sum()) == pages and int(a.table.max()) == pages - 1
    for _ in range(70):                                                              # over a page's end
        x = torch.randn((2, 256), generator=g).bfloat16().cuda()
        assert torch.equal(*(layer(x, c, ids(2, 3), ids(1, 1), 1, 512) for c in (a, b)))


def test_a_full_cache_is_told():
    layer, g = made(4, 2, 64)
    cache = ex.Cache(2, 2, 512, 2, 64)
    x = torch.randn((200, 256), generator=g).bfloat16().cuda()
    with pytest.raises(RuntimeError):
        layer(x, cache, ids(0, 1), ids(100, 100), 100, 512)


def test_gradients_of_the_head_pass():
    """Through autograd: against differences of the loss in 64 bits."""
    D, T, B = 64, 9, 32
    g = torch.Generator().manual_seed(4)
    q, k = torch.randn((T, 3, D), generator=g), torch.randn((T, 1, D), generator=g)
    wq, wk = (1 + 0.2 * torch.randn(D, generator=g) for _ in range(2))
    rq, rk = torch.randn(q.shape, generator=g), torch.randn(k.shape, generator=g)
    angle = torch.arange(32)[:, None] * 100.0 ** (-torch.arange(D // 2) * 2.0 / D)
    cos, sin, pos = angle.cos().contiguous(), angle.sin().contiguous(), torch.randint(0, 32, (T,), generator=g)
    leaves = [t.cuda().requires_grad_() for t in (q, k, wq, wk)]
    q2, k2 = ex.HeadNorms.apply(*leaves, cos.cuda(), sin.cuda(), pos.cuda(), B)
    ((q2 * rq.cuda()).sum() + (k2 * rk.cuda()).sum()).backward()

    def loss(q, k, wq, wk):
        return float(sum((ref.forward(x, w, 1e-6, cos, sin, pos, False, B)[0] * r.double()).sum() for x, w, r in ((q, wq, rq), (k, wk, rk))))

    for i, t in enumerate((q, k, wq, wk)):
        d = torch.randn(t.shape, generator=g).double()
        args = [x.double() for x in (q, k, wq, wk)]
        step = 1e-6
        up, down = ([x + s * d if j == i else x for j, x in enumerate(args)] for s in (step, -step))
        slope = (loss(*up) - loss(*down)) / (2 * step)
        # 32-bit gradients, each 1e-5 of the largest off at most, summed with d; differences: step^2 and 1e-16 / step of the loss
        grad = leaves[i].grad.cpu().double()
        assert math.isclose(float((grad * d).sum()), slope, abs_tol=1e-5 * float(grad.abs().max() * d.abs().sum()) + 1e-6)


def test_example_runs(capsys):
    cache, y = ex.main(C=256, Hq=4, Hk=2, D=64, steps=3)
    assert cache.lens.tolist() == [0, 0, 34, 304] and y.isfinite().all()
    assert "finite" in capsys.readouterr().out
