"""What the attention side refuses, on the host and before anything is launched (no GPU)."""
import ctypes
from ctypes import byref

import pytest
import torch

import paper_2511_04214_amd as brq
from paper_2511_04214_amd.attention import _Heads, _Rope

OK, NULL, SHAPE, BLOCK, ALIGN, DTYPE = 0, 1, 2, 3, 4, 5
P = 0x1000          # never dereferenced


@pytest.fixture(scope="module")
def L():
    return brq.lib()


def heads(H=4, D=64, p=P, ts=None, hs=None):
    return byref(_Heads(p, H, H * D if ts is None else ts, D if hs is None else hs))


def rope(cos=P, sin=P, pos=P, rows=10, rot=64, inter=0):
    return byref(_Rope(cos, sin, pos, rows, rot, inter))


def test_head_norms(L):
    def fwd(q=heads(), k=heads(1), xdt=1, T=3, D=64, wq=P, wk=P, eps=1e-6, r=rope(), B=32, qo=heads(), ko=heads(1), ydt=1):
        return L.brq_qk_norm_rope(q, k, xdt, T, D, wq, wk, eps, r, B, qo, ko, ydt, None)
    assert fwd(T=0) == OK and fwd(T=0, q=heads(p=None), qo=heads(p=None)) == OK
    assert fwd(q=None) == fwd(qo=None) == fwd(k=None) == fwd(ko=None) == fwd(q=heads(p=None)) == NULL
    assert fwd(r=rope(cos=None)) == fwd(r=rope(sin=None)) == fwd(r=rope(pos=None)) == NULL
    assert fwd(xdt=2) == fwd(ydt=-1) == DTYPE
    for D in (0, 32, 96, 512):
        assert fwd(D=D) == SHAPE
    assert fwd(T=-1) == fwd(eps=-1.0) == fwd(eps=float("nan")) == fwd(T=1 << 40) == fwd(qo=heads(3)) == SHAPE
    assert fwd(q=heads(0)) == fwd(r=rope(rot=128)) == fwd(r=rope(rot=8)) == fwd(r=rope(rot=0)) == fwd(r=rope(rows=0)) == SHAPE
    assert fwd(q=heads(ts=-64)) == fwd(q=heads(hs=-64)) == SHAPE
    assert fwd(qo=heads(ts=0)) == fwd(qo=heads(hs=0)) == fwd(qo=heads(ts=128)) == SHAPE       # an output that overlaps itself
    assert fwd(q=heads(p=P + 8)) == fwd(q=heads(ts=260)) == fwd(q=heads(hs=68)) == fwd(qo=heads(hs=68, ts=400)) == ALIGN
    assert fwd(r=rope(cos=P + 4)) == fwd(r=rope(pos=P + 4)) == fwd(wq=P + 2) == ALIGN
    for B in (0, 2, 4, 24, 128):
        assert fwd(B=B) == BLOCK

    def back(q=heads(), k=heads(1), T=3, D=64, wq=P, wk=P, B=32, gq=heads(), gk=heads(1), gdt=0, dq=heads(), dk=heads(1), dwq=P, dwk=P, ws=P, n=1 << 30):
        return L.brq_qk_norm_rope_backward(q, k, 1, T, D, wq, wk, 1e-6, rope(), B, gq, gk, gdt, dq, dk, dwq, dwk, ws, n, None)
    assert back(gq=None) == back(gk=None) == back(dq=None) == back(dk=None) == back(k=None) == back(ws=None) == NULL
    assert back(wq=None) == back(wk=None) == NULL                                             # a gradient of a weight that is not there
    assert back(n=16) == back(gq=heads(5)) == back(dk=heads(2)) == back(dq=heads(ts=0)) == SHAPE
    assert back(gdt=3) == DTYPE and back(B=3) == BLOCK and back(ws=P + 8) == back(dwq=P + 1) == ALIGN
    assert back(T=0, dwq=None, dwk=None, ws=None, n=0) == OK
    n = ctypes.c_int64()
    assert L.brq_qk_norm_rope_backward_workspace(3, 4, 1, 64, None) == NULL
    assert L.brq_qk_norm_rope_backward_workspace(3, 4, 1, 65, byref(n)) == L.brq_qk_norm_rope_backward_workspace(-1, 4, 1, 64, byref(n)) == SHAPE
    assert brq.qk_norm_rope_backward_workspace(0, 4, 1, 64) == 0 < brq.qk_norm_rope_backward_workspace(1, 4, 1, 64)


def test_cache(L):
    def app(q=heads(), k=heads(2), v=heads(2), xdt=1, T=3, D=64, r=rope(), B=32, Bv=64, slots=P, pool=P, pages=5, qo=heads()):
        return L.brq_kv4_append(q, k, v, xdt, T, D, P, P, 1e-6, r, B, Bv, slots, pool, pages, qo, None)
    assert app(T=0) == OK and app(T=0, q=None, qo=None, slots=None, pool=None, pages=0) == OK
    assert app(k=None) == app(v=None) == app(q=None) == app(qo=None) == app(slots=None) == app(pool=None) == NULL
    assert app(D=256) == app(v=heads(1)) == app(pages=-1) == app(T=-2) == SHAPE
    assert app(B=128) == app(Bv=5) == BLOCK and app(xdt=9) == DTYPE and app(pool=P + 8) == app(slots=P + 4) == app(v=heads(2, p=P + 2)) == ALIGN

    def read(pool=P, pages=5, T=3, D=64, slots=P, k=heads(2), v=heads(2), ydt=1):
        return L.brq_kv4_read(pool, pages, T, D, slots, k, v, ydt, None)
    assert read(T=0) == OK and read(k=None) == read(v=None) == read(slots=None) == read(pool=None) == NULL
    assert read(D=32) == read(v=heads(3)) == read(T=-1) == read(k=heads(2, ts=0)) == SHAPE and read(ydt=4) == DTYPE and read(pool=P + 1) == ALIGN
    n = ctypes.c_int64()
    assert L.brq_kv4_page_bytes(0, 64, byref(n)) == L.brq_kv4_page_bytes(1, 32, byref(n)) == SHAPE and L.brq_kv4_page_bytes(1, 64, None) == NULL
    assert brq.kv4_page_bytes(8, 128) == 8 * 68 * 128


def test_attention(L):
    def att(q=heads(8), T=6, D=64, pool=P, pages=9, Hk=2, table=P, cols=4, lens=P, cu=P, S=3, causal=1, window=0, max_q=4, max_kv=256, out=heads(8), lse=P, ws=P, n=1 << 40):
        return L.brq_kv4_attention(q, T, D, pool, pages, Hk, table, cols, lens, cu, S, 0.125, causal, window, max_q, max_kv, out, lse, ws, n, None)
    assert att(T=0) == OK and att(S=0) == OK
    assert att(q=None) == att(out=None) == att(pool=None) == att(table=None) == att(lens=None) == NULL
    assert att(D=96) == att(D=256) == att(Hk=3) == att(Hk=0) == att(out=heads(4)) == att(cu=None) == att(window=-1) == att(window=5, causal=0) == SHAPE
    assert att(max_q=0) == att(max_kv=-1) == att(cols=-1) == att(T=-1) == att(S=-1) == att(S=1 << 30) == att(out=heads(8, ts=0)) == SHAPE
    assert att(pool=P + 8) == att(lens=P + 2) == att(cu=P + 1) == att(lse=P + 2) == att(ws=P + 4) == att(q=heads(8, p=P + 4)) == ALIGN
    n = ctypes.c_int64()
    assert L.brq_kv4_attention_workspace(6, 3, 8, 2, 64, 4, 256, None) == NULL
    assert L.brq_kv4_attention_workspace(6, 3, 8, 3, 64, 4, 256, byref(n)) == SHAPE


def test_pages(L):
    n = ctypes.c_int64()
    assert L.brq_kv4_pages_workspace(3, 10, None) == NULL and L.brq_kv4_pages_workspace(-1, 10, byref(n)) == SHAPE
    assert L.brq_kv4_pages_copy(P, 64, 5, P, P, 0, None) == OK
    assert L.brq_kv4_pages_copy(None, 64, 5, P, P, 2, None) == L.brq_kv4_pages_copy(P, 64, 5, None, P, 2, None) == NULL
    assert L.brq_kv4_pages_copy(P, 40, 5, P, P, 2, None) == L.brq_kv4_pages_copy(P, 64, -1, P, P, 2, None) == SHAPE
    assert L.brq_kv4_pages_copy(P + 8, 64, 5, P, P, 2, None) == L.brq_kv4_pages_copy(P, 64, 5, P + 2, P, 2, None) == ALIGN

    def fork(pool=P, pb=64, pages=5, table=P, S=4, cols=3, lens=P, refs=P, a=P, b=P, n=2, failed=P, ws=P):
        return L.brq_kv4_pages_fork(pool, pb, pages, table, S, cols, lens, refs, a, b, n, failed, ws, None)
    assert fork(pool=None) == fork(table=None) == fork(lens=None) == fork(refs=None) == fork(a=None) == fork(b=None) == fork(failed=None) == fork(ws=None) == NULL
    assert fork(S=-1) == fork(cols=-1) == fork(n=-1) == fork(S=1 << 20, cols=1 << 20) == fork(pb=8) == SHAPE
    assert fork(ws=P + 4) == fork(failed=P + 1) == fork(refs=P + 2) == ALIGN
    assert L.brq_kv4_pages_free(P, 4, 3, P, P, 5, P, 0, None) == OK and L.brq_kv4_pages_free(P, 4, 3, P, P, 5, None, 2, None) == NULL
    assert L.brq_kv4_pages_free(P, 4, -3, P, P, 5, P, 2, None) == SHAPE and L.brq_kv4_pages_free(P, 4, 3, P + 1, P, 5, P, 2, None) == ALIGN
    assert L.brq_kv4_pages_reserve(P, 4, 3, P, 5, P, None, 2, P, P, None) == L.brq_kv4_pages_reserve(P, 4, 3, P, 5, P, P, 2, None, P, None) == NULL
    assert L.brq_kv4_pages_reserve(P, -4, 3, P, 5, P, P, 2, P, P, None) == SHAPE
    assert L.brq_kv4_pages_compact(P, 64, 5, P, 4, 3, None, P, P, None) == L.brq_kv4_pages_compact(P, 64, 5, P, 4, 3, P, P, None, None) == NULL
    assert L.brq_kv4_pages_compact(P, 20, 5, P, 4, 3, P, P, P, None) == SHAPE and L.brq_kv4_pages_compact(P, 64, 5, P, 4, 3, P, P, P + 8, None) == ALIGN


def test_the_binding_refuses():
    x, i = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    pool, w = torch.zeros((2, brq.kv4_page_bytes(4, 64)), dtype=torch.uint8), torch.zeros(64)
    for call in (lambda: brq.qk_norm_rope(x, x, w, w), lambda: brq.qk_norm_rope_backward(x, x, x, x, w, w), lambda: brq.kv4_append(pool, i.long(), x, x),
                 lambda: brq.kv4_read(pool, i.long(), 64), lambda: brq.kv4_attention(x, pool, torch.zeros((2, 1), dtype=torch.int32), i),
                 lambda: brq.kv4_pages_copy(pool, i, i), lambda: brq.kv4_pages_fork(pool, torch.zeros((2, 1), dtype=torch.int32), i, i, i, i),
                 lambda: brq.kv4_pages_free(torch.zeros((2, 1), dtype=torch.int32), i, i, i),
                 lambda: brq.kv4_pages_reserve(torch.zeros((2, 1), dtype=torch.int32), i, i, i),
                 lambda: brq.kv4_pages_compact(pool, torch.zeros((2, 1), dtype=torch.int32), i)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()


@pytest.mark.gpu
def test_the_binding_refuses_what_does_not_fit():
    x, f = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 4, 64), device="cuda")
    w, pos, i = torch.zeros(64, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    pool, table = torch.zeros((2, brq.kv4_page_bytes(4, 64)), dtype=torch.uint8, device="cuda"), torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    t = torch.zeros((10, 32), device="cuda")
    for error, call in (
            (ValueError, lambda: brq.qk_norm_rope(x[0], x)), (ValueError, lambda: brq.qk_norm_rope(x, f)), (ValueError, lambda: brq.qk_norm_rope(x, x[:1])),
            (TypeError, lambda: brq.qk_norm_rope(x.half(), None)), (TypeError, lambda: brq.qk_norm_rope(x, None, w.bfloat16())), (ValueError, lambda: brq.qk_norm_rope(x, None, w[:32])),
            (ValueError, lambda: brq.qk_norm_rope(x, None, cos=t, sin=t)), (ValueError, lambda: brq.qk_norm_rope(x, None, cos=t, sin=t, positions=pos[:1])),
            (TypeError, lambda: brq.qk_norm_rope(x, None, cos=t, sin=t, positions=i)), (ValueError, lambda: brq.qk_norm_rope(x, None, cos=t, sin=t[:5], positions=pos)),
            (brq.BrqError, lambda: brq.qk_norm_rope(x, None, B=128)), (ValueError, lambda: brq.qk_norm_rope(x.transpose(1, 2), None)),
            (ValueError, lambda: brq.qk_norm_rope_backward(x, x, x, None)), (ValueError, lambda: brq.qk_norm_rope_backward(x, None, x[:, :2], None)),
            (ValueError, lambda: brq.kv4_append(pool[:, :-1].contiguous(), pos, x, x)), (ValueError, lambda: brq.kv4_append(pool, pos, x, f)),
            (TypeError, lambda: brq.kv4_append(pool, i, x, x)), (ValueError, lambda: brq.kv4_read(pool, pos, 80)),
            (TypeError, lambda: brq.kv4_attention(f, pool, table, i)), (ValueError, lambda: brq.kv4_attention(x, pool, table[:1], i[:1])),
            (TypeError, lambda: brq.kv4_attention(x, pool, table.long(), i)), (brq.BrqError, lambda: brq.kv4_attention(x, pool, table, i, causal=False, window=3)),
            (brq.BrqError, lambda: brq.kv4_attention(x[:, :3], pool, table, i)), (ValueError, lambda: brq.kv4_pages_fork(pool, table, i, i[:1], i, i)),
            (ValueError, lambda: brq.kv4_pages_fork(pool, table, i, i, i, i[:1])), (TypeError, lambda: brq.kv4_pages_free(table, i, i, pos)),
            (ValueError, lambda: brq.kv4_pages_compact(pool, table, i, workspace=torch.zeros(4, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(error):
            call()
