"""Plain 64-bit implementations (CPU, torch) of the attention side, written from the formulas of include/brq_attn.h."""
import math

import torch

F64 = torch.float64
GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64)


def hadamard(B):
    h = torch.ones((1, 1), dtype=F64)
    while h.shape[0] < B:
        h = torch.cat((torch.cat((h, h), 1), torch.cat((h, -h), 1)), 0)
    return h / math.sqrt(B)


def rotate(x, B):
    return x if B == 1 else (x.reshape(-1, B) @ hadamard(B)).reshape(x.shape)


def spread(x, B):
    """What bounds every intermediate of a rotation of values of magnitude x."""
    return x.abs() if B == 1 else (x.abs().reshape(-1, B).sum(-1, keepdim=True) / math.sqrt(B)).expand(-1, B).reshape(x.shape)


def turn(x, cos, sin, positions, interleaved, sign=1.0, magnitude=False):
    if cos is None:
        return x
    rot, half = cos.shape[1] * 2, cos.shape[1]
    c, s = cos.double()[positions][:, None], sign * sin.double()[positions][:, None]
    y = x.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
    if magnitude:
        c, s = c.abs(), s.abs()
        y[..., a], y[..., b] = x[..., a] * c + x[..., b] * s, x[..., b] * c + x[..., a] * s
    else:
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y


def norm(x, w, eps):
    return x if w is None else x / torch.sqrt(x.pow(2).mean(-1, keepdim=True) + eps) * w.double()


def forward(x, w, eps, cos, sin, positions, interleaved, B):
    """(y, bound on its magnitude's intermediates)"""
    n = norm(x.double(), w, eps)
    return (rotate(turn(n, cos, sin, positions, interleaved), B),
            spread(turn(n.abs(), cos, sin, positions, interleaved, magnitude=True), B))


def backward(x, g, w, eps, cos, sin, positions, interleaved, B):
    """(dx, bound, dw, bound)"""
    gn = turn(rotate(g.double(), B), cos, sin, positions, interleaved, sign=-1.0)
    gm = turn(spread(g.double(), B), cos, sin, positions, interleaved, magnitude=True)
    if w is None:
        return gn, gm, None, None
    r = 1 / torch.sqrt(x.double().pow(2).mean(-1, keepdim=True) + eps)
    u, wd = x.double() * r, w.double()
    y, ym = gn * wd, gm * wd.abs()
    dx = r * (y - u * (y * u).mean(-1, keepdim=True))
    return dx, r * (ym + u.abs() * (ym * u.abs()).mean(-1, keepdim=True)), (gn * u).sum((0, 1)), (gm * u.abs()).sum((0, 1))


def code_values(codes, scales):
    """Row-major codes [..., K / 2] and scale bytes [..., K / 32] -> values."""
    c = codes.long()
    v = torch.stack((c & 15, c >> 4), -1).flatten(-2)
    v = GRID[v & 7] * (1 - 2 * (v >> 3))
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def page_index(D):
    """Byte offsets inside a head of a page: keys' codes [64, D / 2], scales [64, D / 32], values' codes and scales."""
    t, j, n, P = torch.arange(64)[:, None], torch.arange(D // 2)[None], torch.arange(D // 32)[None], D // 32
    return (t * (D // 2) + j, 32 * D + (n * 16 + t % 16) * 4 + t // 16,
            34 * D + ((t // 4 * 16 + j // P) * 4 + t % 4) * P + j % P, 66 * D + ((t // 4 % 4 * P + n) * 4 + t // 16) * 4 + t % 4)


def cache_values(pool, Hk, D):
    """All keys and values of a cache [pages, Hk * 68 D] (CPU): [pages, 64, Hk, D] each."""
    heads = pool.view(pool.shape[0], Hk, 68 * D)
    kc, ks, vc, vs = page_index(D)
    return [code_values(heads[..., c], heads[..., s]).transpose(1, 2) for c, s in ((kc, ks), (vc, vs))]


def attention(q, values, table, lens, scale, causal, window, cu_q, max_q, max_kv):
    """(out, lse, sum of p |v|, largest error of a score) of rows that are somebody's; NaN in the others."""
    k, v = values
    T, Hq, D = q.shape
    G = Hq // k.shape[2]
    out, lse = torch.full((T, Hq, D), math.nan, dtype=F64), torch.full((T, Hq), math.nan, dtype=F64)
    mag, ds = torch.zeros((T, Hq, D), dtype=F64), torch.zeros((T, Hq), dtype=F64)
    for s in range(table.shape[0]):
        q0, q1 = (s, s + 1) if cu_q is None else (int(cu_q[s]), int(cu_q[s + 1]))
        n = int(lens[s])
        seen = min(n, max_kv, table.shape[1] * 64)
        pages = table[s, : (max(0, seen) + 63) // 64].long()
        ok = (pages >= 0) & (pages < k.shape[0])
        kk, vv = (x[pages.clamp(0, k.shape[0] - 1)].reshape(-1, x.shape[2], D)[: max(0, seen)] for x in (k, v))
        real = ok.repeat_interleave(64)[: max(0, seen)]
        j = torch.arange(max(0, seen))
        for i in range(min(q1 - q0, max_q)):
            p = n - (q1 - q0) + i
            see = real.clone()
            if causal:
                see &= j <= p
                if window:
                    see &= j > p - window
            x = q[q0 + i].double()
            if not see.any():
                out[q0 + i], lse[q0 + i] = 0.0, -math.inf
                continue
            ks, vs = kk[see], vv[see]
            for h in range(Hq):
                a = ks[:, h // G] @ x[h] * scale
                w = torch.softmax(a, 0)
                out[q0 + i, h], lse[q0 + i, h] = w @ vs[:, h // G], torch.logsumexp(a, 0)
                mag[q0 + i, h] = w @ vs[:, h // G].abs()
                # a query's two terms, and a sum of D products and the multiplication by the scale in 32 bits
                ds[q0 + i, h] = abs(scale) * float((ks[:, h // G].abs().sum(1) * x[h].abs().max() * 2.0 ** -19
                                                   + ks[:, h // G].abs() @ x[h].abs() * (D + 4) * 2.0 ** -24).max())
    return out, lse, mag, ds
