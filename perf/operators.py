"""What the attention side of the library is timed on: the passes its users make, over the sizes they make them at.

Four operators, and a pass through two of them as a decoding layer makes it:

  heads      qk_norm_rope and its backward: RMS norm of every query and key head, position rotation, block rotation
  append     kv4_append (then kv4_read): the same in front of an MXFP4 quantizer that writes keys and values into cache pages
  attention  kv4_attention over such a cache: single tokens, ragged batches, prompts
  step       kv4_append and kv4_attention of one decoding layer
  pages      kv4_pages_fork / _free / _reserve / _compact: what a scheduler does to the pages

With `own` false the same is computed in elementary torch operations in 32 bits; exact() has it in 64.

A cache is one uint8 tensor [pages, 68 * D * Hk]: a page holds 64 tokens, a head of it 68 * D bytes: key codes [64][D / 2],
key scales, value codes, value scales, in the orders that _unpack() spells out.
"""
import math
import random

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_PAGE = 64
_EPS = 1e-6
_THETA = 500000.0


# ---- cases

def _heads(name, T, Hq, Hk, D, dtype="bf16", rot=None, interleaved=False, B=1, norm=True):
    c = dict(kind="heads", T=T, Hq=Hq, Hk=Hk, D=D, dtype=dtype, rot=D if rot is None else rot, interleaved=interleaved, B=B, norm=norm)
    return dict(c, name=name) if name else c


def _append(name, T, Hq, Hk, D, B=32, Bv=32, norm=True, dtype="bf16"):
    c = dict(kind="append", T=T, Hq=Hq, Hk=Hk, D=D, B=B, Bv=Bv, norm=norm, dtype=dtype, rot=D, interleaved=False)
    return dict(c, name=name) if name else c


def _attention(name, S, q, L, Hq, Hk, D, ragged=True, causal=True, window=0, lens_seed=0):
    c = dict(kind="attention", S=S, q=q, L=L, Hq=Hq, Hk=Hk, D=D, ragged=ragged, causal=causal, window=window, lens_seed=lens_seed)
    return dict(c, name=name) if name else c


def _step(name, S, L, Hq, Hk, D, lens_seed=0):
    c = dict(kind="step", S=S, q=1, L=L, Hq=Hq, Hk=Hk, D=D, ragged=S > 1, causal=True, window=0, lens_seed=lens_seed, B=32, Bv=32,
             norm=True, dtype="bf16", rot=D, interleaved=False)
    return dict(c, name=name) if name else c


def _pages(name, what, S, L, Hk, D, lens_seed=0):
    c = dict(kind="pages", what=what, S=S, L=L, Hk=Hk, D=D, lens_seed=lens_seed)
    return dict(c, name=name) if name else c


def listed():
    return [
        # fine-tuning: 8192 tokens of a layer with 4096 channels in 32 heads and 8 shared key heads, forward and backward
        _heads("heads_train_8192", 8192, 32, 8, 128, B=32),
        # a small model's heads in 32 bits: odd counts, half of the channels turned, neighbouring channels as pairs
        _heads("heads_f32_odd", 333, 7, 1, 64, dtype="f32", rot=32, interleaved=True),
        # a prompt's keys and values go into the cache
        _append("append_prompt_4096", 4096, 32, 8, 128),
        # ... and those of a ragged batch of decoding sequences, nothing normalised, heads of 64
        _append("append_decode_100", 100, 32, 8, 64, norm=False, B=64, Bv=64),
        # generation of one short sequence: latency
        _attention("decode_1_short", 1, 1, 100, 32, 8, 128),
        # generation of one sequence with a long context
        _attention("decode_1_long", 1, 1, 131072, 32, 8, 128, ragged=False),
        # generation of a ragged batch
        _attention("decode_batch_100", 100, 1, 8192, 32, 8, 128, lens_seed=3),
        # a prompt of 8192 tokens over its own cache
        _attention("prompt_8192", 1, 8192, 8192, 32, 8, 128, ragged=False),
        # chunks of several prompts, ragged, over what came before, in a window of 1024, heads of 64
        _attention("chunks_window_6", 6, 500, 4000, 16, 4, 64, window=1024, lens_seed=5),
        # one layer's decoding step of 16 sequences: the new keys and values go in, attention reads all
        _step("step_16", 16, 2000, 32, 8, 128),
        # 48 sequences are forked, their parents freed and the children given room for 100 tokens more
        _pages("pages_fork_48", "fork", 48, 1000, 8, 128),
        # a cache with half of its sequences gone is made dense
        _pages("pages_compact_96", "compact", 96, 2500, 8, 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "append", "attention", "attention", "attention", "step", "pages"])
    D = rng.choice([64, 128, 128])
    Hk = rng.choice([1, 2, 4, 8, 8])
    Hq = Hk * rng.choice([1, 2, 4, 4, 5, 8])
    Hq = min(Hq, 32 // Hk * Hk)
    if kind == "heads":
        return _heads(None, _log(rng, 1, 8192), Hq, Hk, D, dtype=rng.choice(["bf16", "bf16", "f32"]), rot=rng.choice([D, D, D // 2]),
                      interleaved=rng.random() < 0.3, B=rng.choice([1, 32, D]), norm=rng.random() < 0.8)
    if kind == "append":
        return _append(None, _log(rng, 1, 4096), Hq, Hk, D, B=rng.choice([1, 32, D]), Bv=rng.choice([1, 32, D]), norm=rng.random() < 0.7,
                       dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind == "attention":
        s = rng.randrange(1 << 20)
        window = rng.choice([0, 0, 0, 256, 1000])
        if rng.random() < 0.55:                     # single tokens
            S = _log(rng, 1, 128)
            return _attention(None, S, 1, max(1, _log(rng, 1, min(131072, 800000 // S))), Hq, Hk, D, window=window, lens_seed=s)
        S = _log(rng, 1, 8)
        q = _log(rng, 2, 8192 // S)
        L = q if rng.random() < 0.4 else max(q, _log(rng, q, max(q, 8192 // S)))
        return _attention(None, S, q, L, Hq, Hk, D, window=window, causal=rng.random() < 0.85 or window > 0, lens_seed=s)
    if kind == "step":
        S = _log(rng, 1, 100)
        return _step(None, S, max(1, _log(rng, 1, 400000 // S)), Hq, Hk, D, lens_seed=rng.randrange(1 << 20))
    S = _log(rng, 2, 128)
    return _pages(None, rng.choice(["fork", "compact"]), S, _log(rng, 10, min(8192, 240000 // S)), Hk, D, lens_seed=rng.randrange(1 << 20))


def _lens(c):
    """(query lengths, context lengths) of the sequences: the case's own, whatever the seed of its values."""
    r = random.Random(c["lens_seed"] * 7919 + c["S"] * 131 + c["L"])
    S, L, q = c["S"], c["L"], c.get("q", 1)
    if not c.get("ragged", True):
        return [q] * S, [L] * S
    ctx = [r.randint((L + 1) // 2, L) if r.random() < 0.7 else r.randint(0, L) for _ in range(S)]
    ctx[r.randrange(S)] = L
    if c["kind"] == "step":
        ctx = [max(1, n) for n in ctx]
    qs = [q] * S if q == 1 else [r.randint(1, q) for _ in range(S)]
    if q > 1:
        qs[r.randrange(S)] = q
    return qs, ctx


def _visible(c, q, n):
    """Keys that the q queries at the end of a context of n see, all together."""
    if not c["causal"]:
        return q * n
    p = torch.arange(n - q, n, dtype=torch.int64)
    hi = (p + 1).clamp(0, n)
    lo = (p - c["window"] + 1).clamp(min=0) if c["window"] else torch.zeros_like(p)
    return int((hi - torch.minimum(lo, hi)).sum())


def _read_tokens(c, q, n):
    """Tokens of a context of n that the q queries at its end have to read."""
    if not c["causal"] or not c["window"]:
        return n
    return min(n, q + c["window"] - 1)


def work(case):
    c = case
    if c["kind"] == "heads":                        # x, y, then x, g, dx
        es = 2 if c["dtype"] == "bf16" else 4
        n = c["T"] * (c["Hq"] + c["Hk"]) * c["D"]
        return {"bytes": n * es * 5 + c["T"] * c["rot"] * 4 * 2, "flops": 30 * n}
    kv = c["Hk"] * c["D"] * 17 // 16                # bytes of a token's keys and values in the cache
    if c["kind"] == "append":                       # q, k, v in; q out; the cache's bytes written and read back; values out
        es = 2 if c["dtype"] == "bf16" else 4
        n = c["T"] * c["D"]
        return {"bytes": n * es * (2 * c["Hq"] + 2 * c["Hk"]) + c["T"] * (2 * kv + c["rot"] * 4) + 2 * n * c["Hk"] * 2, "flops": 30 * n * (c["Hq"] + 2 * c["Hk"])}
    if c["kind"] == "pages":
        page = kv * _PAGE
        qs, ctx = _lens(c)
        if c["what"] == "fork":                     # the last page of each, if it is not full
            return {"bytes": 2 * page * sum(n % _PAGE > 0 for n in ctx) + 2 * 4 * sum(-(-n // _PAGE) for n in ctx), "flops": 0}
        live = sum(-(-n // _PAGE) for n in ctx[::2])
        gone = sum(-(-n // _PAGE) for n in ctx[1::2])
        return {"bytes": 2 * page * (live * gone // max(1, live + gone)) + 8 * (live + gone), "flops": 0}
    qs, ctx = _lens(c)
    T = sum(qs)
    b = sum(_read_tokens(c, q, n) for q, n in zip(qs, ctx)) * kv + T * c["Hq"] * (c["D"] * 4 + (4 if c["kind"] == "attention" else 0))
    f = 4 * c["D"] * c["Hq"] * sum(_visible(c, q, n) for q, n in zip(qs, ctx))
    if c["kind"] == "step":
        b += T * c["D"] * 2 * (c["Hq"] + 2 * c["Hk"])
    return {"bytes": b, "flops": f}


# ---- inputs

def _rand(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _qkv(g, c, T):
    """Rows of a packed projection, [T, Hq + 2 Hk, D]: a few channels of queries and keys far larger than the rest, values even."""
    x = _rand(g, T, c["Hq"] + 2 * c["Hk"], c["D"])
    big = torch.randperm(c["D"], generator=g, device="cuda")[: c["D"] // 16]
    x[:, : c["Hq"] + c["Hk"]][..., big] *= 8.0
    return x.to(_DTYPES[c.get("dtype", "bf16")])


def _rope_tables(positions, rot):
    f = _THETA ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    a = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * f
    return a.cos().float(), a.sin().float()


def _pool(g, pages, Hk, D):
    """A cache of plausible content: codes of a rounded normal distribution, scales of a few binades about one (keys) and an eighth (values)."""
    nk, ns = 32 * D, 2 * D
    pool = torch.empty((pages, Hk, 68 * D), dtype=torch.uint8, device="cuda")
    # codes by the share of a normal value scaled to a largest of about 2.4 times its deviation
    table = torch.tensor([c | s for c, n in zip(range(8), (38, 68, 56, 40, 30, 17, 6, 1)) for s in (0, 8) for _ in range(n // 2 + (s and n % 2))],
                         dtype=torch.uint8, device="cuda")
    for at, e in ((0, 126), (nk + ns, 123)):
        r = torch.randint(0, table.numel() ** 2, (pages, Hk, nk), generator=g, device="cuda", dtype=torch.int32)
        code = table[r % table.numel()] | (table[r // table.numel()] << 4)
        pool[:, :, at: at + nk] = torch.where((code & 7) == 0, code & 0xF0, code) & torch.where((code & 0x70) == 0, 0x0F, 0xFF).to(torch.uint8)
        pool[:, :, at + nk: at + nk + ns] = torch.randint(e - 1, e + 2, (pages, Hk, ns), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    return pool.view(pages, Hk * 68 * D)


def _tables(g, ctx, cols, pages):
    """Page tables: every sequence's pages anywhere in the cache, -1 where it has none."""
    need = torch.tensor([-(-n // _PAGE) for n in ctx], device="cuda")
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(cols, device="cuda")
    start = need.cumsum(0) - need
    at = (start[:, None] + col).clamp(max=pages - 1)
    return torch.where(col < need[:, None], perm[at], -1).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=c)
    if c["kind"] == "heads" or c["kind"] == "append" or c["kind"] == "step":
        T = c["S"] if c["kind"] == "step" else c["T"]
        D, Hq, Hk = c["D"], c["Hq"], c["Hk"]
        x = _qkv(g, c, T)
        s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq: Hq + Hk], x[:, Hq + Hk:]
        s["wq"] = (1 + 0.3 * _rand(g, D)) if c["norm"] else None
        s["wk"] = (1 + 0.3 * _rand(g, D)) if c["norm"] else None
        top = 8192 if c["kind"] != "step" else c["L"]
        s["cos"], s["sin"] = _rope_tables(top, c["rot"])
        s["pos"] = torch.randint(0, top, (T,), generator=g, device="cuda")
    if c["kind"] == "heads":
        s["gq"] = _rand(g, T, Hq, D).to(x.dtype)
        s["gk"] = _rand(g, T, Hk, D).to(x.dtype)
        return s
    if c["kind"] == "append":
        pages = -(-T // _PAGE) + 8
        s["pool"] = _pool(g, pages, Hk, D)
        s["slots"] = torch.randperm(pages * _PAGE, generator=g, device="cuda")[:T]
        return s
    qs, ctx = _lens(c)
    S, D, Hk = c["S"], c["D"], c["Hk"]
    if c["kind"] == "pages":
        need = [-(-n // _PAGE) for n in ctx]
        used = sum(need)
        pages = used + (3 * S + 8 if c["what"] == "fork" else used // 8)
        seqs = 2 * S if c["what"] == "fork" else S
        cols = max(need) + 4
        s["pool"] = torch.randint(0, 256, (pages, Hk * 68 * D), generator=g, device="cuda", dtype=torch.uint8)
        table = _tables(g, ctx, cols, pages)
        s["table"] = torch.cat([table, torch.full((seqs - S, cols), -1, dtype=torch.int32, device="cuda")])
        s["lens"] = torch.tensor(ctx + [0] * (seqs - S), dtype=torch.int32, device="cuda")
        refs = torch.zeros(pages + 1, dtype=torch.int32, device="cuda")
        refs.scatter_add_(0, torch.where(table < 0, pages, table).flatten().long(), torch.ones(table.numel(), dtype=torch.int32, device="cuda"))
        s["refs"] = refs[:pages].contiguous()
        s["parents"] = torch.arange(S, dtype=torch.int32, device="cuda")
        s["children"] = torch.arange(S, 2 * S, dtype=torch.int32, device="cuda")
        s["gone"] = torch.arange(1, S, 2, dtype=torch.int32, device="cuda")
        s["more"] = torch.tensor([n + 100 for n in ctx], dtype=torch.int32, device="cuda")
        return s
    used = sum(-(-n // _PAGE) for n in ctx)
    s["pool"] = _pool(g, used + 4, Hk, D)
    cols = -(-c["L"] // _PAGE)
    s["table"] = _tables(g, ctx, cols, used + 4)
    s["lens"] = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    s["scale"] = D ** -0.5
    s["max_q"], s["max_kv"] = max(qs), c["L"]
    if c["kind"] == "step":
        s["pos"] = (s["lens"] - 1).long()
        s["slots"] = s["table"].gather(1, (s["pos"] // _PAGE)[:, None])[:, 0].long() * _PAGE + s["pos"] % _PAGE
        return s
    T = sum(qs)
    s["q"] = (_rand(g, T, c["Hq"], D) * 2.0).to(torch.bfloat16)
    s["cu_q"] = None if c["q"] == 1 else torch.tensor([0] + qs, dtype=torch.int32, device="cuda").cumsum(0).to(torch.int32)
    return s


# ---- the plain forms: elementary operations, 32 bits

def _hadamard(B, like):
    i = torch.arange(B, device=like.device)
    bits = i[:, None] & i[None, :]
    odd = (bits ^ (bits >> 4) ^ (bits >> 8)) & 15
    odd = odd ^ (odd >> 2)
    odd = (odd ^ (odd >> 1)) & 1
    return (1 - 2 * odd).to(like.dtype) * B ** -0.5


def _rotate(x, B):
    if B == 1:
        return x
    return (x.reshape(-1, B) @ _hadamard(B, x)).reshape(x.shape)


def _turn(x, cos, sin, rot, interleaved):
    h, rest = x[..., :rot], x[..., rot:]
    a, b = (h[..., 0::2], h[..., 1::2]) if interleaved else (h[..., : rot // 2], h[..., rot // 2:])
    y, z = a * cos - b * sin, b * cos + a * sin
    y = torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1)
    return torch.cat((y, rest), -1)


def _normed(x, w):
    return x if w is None else x * (x.square().mean(-1, keepdim=True) + _EPS).rsqrt() * w


def _head_path(s, x, w):
    c = s["case"]
    cos, sin = s["cos"][s["pos"]][:, None], s["sin"][s["pos"]][:, None]
    return _rotate(_turn(_normed(x.float(), w), cos, sin, c["rot"], c["interleaved"]), c["B"])


def _head_grads(s, x, w, g):
    c = s["case"]
    cos, sin = s["cos"][s["pos"]][:, None], s["sin"][s["pos"]][:, None]
    n = _turn(_rotate(g.float(), c["B"]), cos, -sin, c["rot"], c["interleaved"])
    if w is None:
        return n, None
    x = x.float()
    r = (x.square().mean(-1, keepdim=True) + _EPS).rsqrt()
    y = n * w
    return r * (y - x * (r * r) * (y * x).mean(-1, keepdim=True)), (n * x * r).sum((0, 1))


def _e2m1(x):
    """Codes of the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 (ties to the even code), no sign on zero."""
    m = x.abs()
    edges = ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True))
    code = sum(((m > e) if even else (m >= e)).to(torch.int32) for e, even in edges)
    return code + 8 * ((x < 0) & (code > 0)).to(torch.int32)


def _quantized(x):
    """(codes, scale bytes) of groups of 32 along the last axis: scale 2^(floor(log2 of the largest) - 2)."""
    g = x.reshape(*x.shape[:-1], -1, 32)
    e = (((g.abs().amax(-1).view(torch.int32) >> 23) & 255) - 2).clamp(min=0)
    y = torch.ldexp(g, 127 - e.unsqueeze(-1))
    return _e2m1(y).reshape(x.shape), e


def _values(codes, e):
    lut = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    v = lut[(codes & 7).long()] * (1 - 2 * (codes >> 3)).float()
    return torch.ldexp(v, (e.int() - 127).repeat_interleave(32, -1))


def _slot_bytes(slots, Hk, D):
    """Where the code bytes and scale bytes of tokens at `slots` are in the cache: [T, Hk, D / 2] and [T, Hk, D / 32], keys then values."""
    page, t = slots // _PAGE, slots % _PAGE
    h = torch.arange(Hk, device=slots.device)
    base = (page[:, None] * Hk + h)[..., None] * (68 * D)
    t = t[:, None, None]
    j, n = torch.arange(D // 2, device=slots.device), torch.arange(D // 32, device=slots.device)
    per = D // 32                                   # code bytes of one of 16 columns
    kc = base + t * (D // 2) + j
    ks = base + 32 * D + (n * 16 + t % 16) * 4 + t // 16
    vc = base + 34 * D + ((t // 4 * 16 + j // per) * 4 + t % 4) * per + j % per
    vs = base + 66 * D + ((t // 4 % 4 * (D // 32) + n) * 4 + t // 16) * 4 + t % 4
    return kc, ks, vc, vs


def _unpack(pages, D):
    """Cache pages [..., Hk, 68 D] as values: keys and values [..., 64, Hk, D]."""
    lead, G = pages.shape[:-1], D // 32
    kc = pages[..., : 32 * D].reshape(*lead, 64, D // 2)
    ks = pages[..., 32 * D: 34 * D].reshape(*lead, G, 16, 4).movedim(-3, -1).movedim(-2, -3).reshape(*lead, 64, G)
    vc = pages[..., 34 * D: 66 * D].reshape(*lead, 16, 16, 4, D // 32).transpose(-3, -2).reshape(*lead, 64, D // 2)
    vs = pages[..., 66 * D:].reshape(*lead, 4, G, 4, 4).movedim(-2, -4).movedim(-1, -2).reshape(*lead, 64, G)
    both = []
    lut = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=pages.device)
    for codes, e in ((kc, ks), (vc, vs)):
        v = torch.stack((lut[(codes & 15).int()], lut[(codes >> 4).int()]), -1).reshape(*lead, 64, G, 32)
        v = v * torch.exp2((e.int() - 127).float()).unsqueeze(-1)
        both.append(v.reshape(*lead, 64, D).movedim(-3, -2))
    return both


def _plain_append(s):
    c = s["case"]
    Hk, D = c["Hk"], c["D"]
    q = _head_path(s, s["q"], s["wq"]).to(s["q"].dtype)
    k, v = _head_path(s, s["k"], s["wk"]), _rotate(s["v"].float(), c["Bv"])
    kc, ks, vc, vs = _slot_bytes(s["slots"], Hk, D)
    flat, out = s["pool"].view(-1), [q]
    for x, at, sat in ((k, kc, ks), (v, vc, vs)):
        codes, e = _quantized(x)
        flat[at] = (codes[..., 0::2] | (codes[..., 1::2] << 4)).to(torch.uint8)
        flat[sat] = e.to(torch.uint8)
        out.append(_values(codes, e).to(torch.bfloat16))
    return out


def _plain_attention(s, q):
    c = s["case"]
    S, D, Hk, Hq, L = c["S"], c["D"], c["Hk"], c["Hq"], s["table"].shape[1] * _PAGE
    G, T = Hq // Hk, q.shape[0]
    cu = s.get("cu_q")
    cu = torch.arange(S + 1, device=q.device) if cu is None else cu.long()
    nq, lens = (cu[1:] - cu[:-1]), s["lens"].long()
    i = torch.arange(s["max_q"], device=q.device)
    row = (cu[:-1, None] + i).clamp(max=T - 1)                                 # [S, Q]: padded with rows of others, dropped below
    real = i < nq[:, None]
    pages = s["pool"].view(-1, Hk, 68 * D)[s["table"].clamp(min=0).long()]
    k, v = (t.reshape(S, L, Hk, D).transpose(1, 2).contiguous() for t in _unpack(pages, D))
    qq = q[row].float().view(S, -1, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(S, Hk, -1, D)
    sc = qq @ k.transpose(2, 3).contiguous()
    sc *= s["scale"]
    j, p = torch.arange(L, device=q.device), (lens - nq)[:, None] + i           # key and query positions
    see = (j < lens[:, None])[:, None]
    if c["causal"]:
        see = see & (j <= p[..., None])
        if c["window"]:
            see = see & (j > p[..., None] - c["window"])
    sc = sc.view(S, Hk, -1, G, L)
    sc.masked_fill_(~see[:, None, :, None], -math.inf)
    m = sc.amax(-1, keepdim=True)
    e = sc.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    z = e.sum(-1, keepdim=True)
    # pages that a table does not have, and tokens past a context's end, hold anything
    v.masked_fill_((j >= lens[:, None])[:, None, :, None], 0.0)
    o = (e.view(S, Hk, -1, L) @ v).view(S, Hk, -1, G, D) / torch.where(z == 0, 1.0, z)
    lse = (m + z.log()).squeeze(-1)
    o, lse = o.permute(0, 2, 1, 3, 4).reshape(S, -1, Hq, D), lse.permute(0, 2, 1, 3).reshape(S, -1, Hq)
    return [o[real].to(q.dtype), lse[real]]


def _plain_fork(s, table, lens, refs):
    pool, par, chi = s["pool"], s["parents"].long(), s["children"].long()
    n, cols = lens[par].long(), table.shape[1]
    full, part = n // _PAGE, n % _PAGE > 0
    col = torch.arange(cols, device=pool.device)
    rows = torch.where(col < full[:, None], table[par], -1)
    shared = torch.where(rows >= 0, rows, pool.shape[0]).flatten().long()
    free = (refs == 0).nonzero()[:, 0]
    new = free[(part.long().cumsum(0) - part.long()).clamp(max=max(0, free.numel() - 1))]
    refs = torch.cat((refs, refs.new_zeros(1))).scatter_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))[:-1]
    rows[part, full[part]] = new[part].int()
    pool[new[part]] = pool[table[par[part], full[part]].long()]
    refs[new[part]] = 1
    table[chi], lens[chi] = rows, lens[par]
    return table, lens, refs


def _plain_free(table, lens, refs, seqs):
    rows = table[seqs.long()]
    at = torch.where(rows >= 0, rows, refs.numel()).flatten().long()
    refs = torch.cat((refs, refs.new_zeros(1))).scatter_add_(0, at, torch.full_like(at, -1, dtype=torch.int32))[:-1]
    table[seqs.long()], lens[seqs.long()] = -1, 0
    return table, lens, refs


def _plain_reserve(table, lens, refs, seqs, more):
    seqs = seqs.long()
    have, want = (lens[seqs].long() + _PAGE - 1) // _PAGE, (more.long() + _PAGE - 1) // _PAGE
    need = (want - have).clamp(min=0)
    first = need.cumsum(0) - need
    col = torch.arange(table.shape[1], device=table.device)
    new = (col >= have[:, None]) & (col < want[:, None])
    free = (refs == 0).nonzero()[:, 0]
    take = free[(first[:, None] + col - have[:, None]).clamp(0, free.numel() - 1)]
    table[seqs] = torch.where(new, take.int(), table[seqs])
    refs[take[new]] = 1
    return table, lens, refs


def _plain_compact(s, table, refs):
    pool = s["pool"]
    live = refs > 0
    L, at = live.sum(), torch.arange(refs.numel(), device=refs.device)
    src, dst = (live & (at >= L)).nonzero()[:, 0], (~live & (at < L)).nonzero()[:, 0]
    to = at.scatter(0, src, dst)
    pool[dst] = pool[src]
    table = torch.where(table >= 0, to[table.clamp(min=0).long()].int(), -1)
    refs = torch.where(at < L, torch.zeros_like(refs).scatter_add_(0, to, torch.where(live, refs, 0)), 0)
    return table, refs, L.int()


# ---- one pass

def _rope_args(s):
    return dict(cos=s["cos"], sin=s["sin"], positions=s["pos"], interleaved=s["case"]["interleaved"])


def run(s):
    c = s["case"]
    if c["kind"] == "heads":
        if not own:
            q, k = (_head_path(s, s[n], s["w" + n]).to(s[n].dtype) for n in "qk")
            (dq, dwq), (dk, dwk) = (_head_grads(s, s[n], s["w" + n], s["g" + n]) for n in "qk")
            return [q, k, dq.to(q.dtype), dk.to(k.dtype), dwq, dwk]
        import paper_2511_04214_amd as brq
        a = dict(wq=s["wq"], wk=s["wk"], eps=_EPS, B=c["B"], **_rope_args(s))
        return [*brq.qk_norm_rope(s["q"], s["k"], **a), *brq.qk_norm_rope_backward(s["q"], s["k"], s["gq"], s["gk"], **a)]
    if c["kind"] == "append" or c["kind"] == "step":
        if own:
            import paper_2511_04214_amd as brq
            q = brq.kv4_append(s["pool"], s["slots"], s["k"], s["v"], q=s["q"], wq=s["wq"], wk=s["wk"], eps=_EPS, B=c["B"], Bv=c["Bv"], **_rope_args(s))
            if c["kind"] == "append":
                return [q, *brq.kv4_read(s["pool"], s["slots"], c["D"])]
            return [q, brq.kv4_attention(q, s["pool"], s["table"], s["lens"], scale=s["scale"], max_kv=s["max_kv"])]
        r = _plain_append(s)
        return r if c["kind"] == "append" else [r[0], _plain_attention(s, r[0])[0]]
    if c["kind"] == "attention":
        if not own:
            return _plain_attention(s, s["q"])
        import paper_2511_04214_amd as brq
        return list(brq.kv4_attention(s["q"], s["pool"], s["table"], s["lens"], scale=s["scale"], causal=c["causal"], window=c["window"],
                                      cu_q=s["cu_q"], max_q=s["max_q"], max_kv=s["max_kv"], want_lse=True))
    # a pass begins with the sequences and counts as they were (the pages' contents come out the same every time)
    table, lens, refs = s["table"].clone(), s["lens"].clone(), s["refs"].clone()
    if not own:
        if c["what"] == "fork":
            table, lens, refs = _plain_fork(s, table, lens, refs)
            table, lens, refs = _plain_free(table, lens, refs, s["parents"])
            table, lens, refs = _plain_reserve(table, lens, refs, s["children"], s["more"])
            return [s["pool"], table, lens, refs]
        table, lens, refs = _plain_free(table, lens, refs, s["gone"])
        table, refs, live = _plain_compact(s, table, refs)
        return [s["pool"], table, lens, refs, live]
    import paper_2511_04214_amd as brq
    if c["what"] == "fork":
        brq.kv4_pages_fork(s["pool"], table, lens, refs, s["parents"], s["children"])
        brq.kv4_pages_free(table, lens, refs, s["parents"])
        brq.kv4_pages_reserve(table, refs, s["children"], s["more"])
        return [s["pool"], table, lens, refs]
    brq.kv4_pages_free(table, lens, refs, s["gone"])
    live = brq.kv4_pages_compact(s["pool"], table, refs)
    return [s["pool"], table, lens, refs, live[0]]


# ---- the definition in 64 bits, one head or sequence at a time

_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_heads(s, x, w, grad=None):
    """y[t, h] = (R_t n(x)) H, with the turn as a D x D matrix for each token; with `grad`, J^T grad and the weight's gradient."""
    c = s["case"]
    T, H, D = x.shape
    H64 = torch.ones((1, 1), dtype=torch.float64, device=x.device)
    while H64.shape[0] < c["B"]:
        H64 = torch.cat((torch.cat((H64, H64), 1), torch.cat((H64, -H64), 1)), 0)
    blocks = torch.block_diag(*[H64 / math.sqrt(c["B"])] * (D // c["B"]))
    half = c["rot"] // 2
    i = torch.arange(half, device=x.device)
    a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
    out, dx, dw = torch.empty((T, H, D), dtype=torch.float64, device=x.device), torch.empty((T, H, D), dtype=torch.float64, device=x.device), 0.0
    for t0 in range(0, T, 1024):
        p = s["pos"][t0: t0 + 1024]
        n = p.numel()
        R = torch.eye(D, dtype=torch.float64, device=x.device).repeat(n, 1, 1)
        co, si = s["cos"][p].double(), s["sin"][p].double()
        R[:, a, a], R[:, b, b], R[:, a, b], R[:, b, a] = co, co, -si, si                  # y_a = a cos - b sin, y_b = a sin + b cos
        M = blocks @ R                                                                    # (blocks are symmetric)
        xs = x[t0: t0 + 1024].double()
        rms = 1.0 if w is None else (xs.pow(2).sum(-1, keepdim=True) / D + _EPS).sqrt()
        u = xs / rms
        wd = torch.ones(D, dtype=torch.float64, device=x.device) if w is None else w.double()
        out[t0: t0 + 1024] = (u * wd) @ M.transpose(1, 2).contiguous()
        if grad is not None:
            gn = grad[t0: t0 + 1024].double() @ M
            gw = gn * wd
            dx[t0: t0 + 1024] = gw if w is None else (gw - u * (gw * u).sum(-1, keepdim=True) / D) / rms
            dw = dw + (gn * u).sum((0, 1))
    return (out, None, None) if grad is None else (out, dx, None if w is None else dw)


def _exact_quantized(x):
    """The value that stands for x in MXFP4, from the definition: nearest grid point, ties to the even code."""
    g = x.reshape(-1, 32)
    top = g.abs().amax(1, keepdim=True)
    e = torch.where(top > 0, torch.floor(torch.log2(torch.where(top > 0, top, 1.0))), -125.0) - 2
    m = (g.abs() / torch.exp2(e)).clamp(max=6.0)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    up = torch.bucketize(m, grid).clamp(1, 7)
    lo, hi = grid[up - 1], grid[up]
    take_hi = (m - lo > hi - m) | ((m - lo == hi - m) & (up % 2 == 0))
    return (torch.where(take_hi, hi, lo) * g.sign() * torch.exp2(e)).reshape(x.shape)


def _exact_cache(pool, Hk, D, table_row, n):
    """Keys and values [Hk, n, D] of one sequence in 64 bits, byte by byte from the layout's formulas."""
    t = torch.arange(n, device=pool.device)
    at = _slot_bytes(table_row.long()[t // _PAGE] * _PAGE + t % _PAGE, Hk, D)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=pool.device)
    flat, got = pool.view(-1), []
    for codes, scales in (at[:2], at[2:]):
        b, e = flat[codes].long(), flat[scales].double() - 127
        v = torch.empty((n, Hk, D), dtype=torch.float64, device=pool.device)
        v[..., 0::2] = grid[b % 8] * (1 - 2 * (b // 8 % 2))
        v[..., 1::2] = grid[b // 16 % 8] * (1 - 2 * (b // 128))
        got.append((v.view(n, Hk, -1, 32) * torch.exp2(e)[..., None]).view(n, Hk, D).transpose(0, 1))
    return got


def _exact_attention(s, q, keys_values):
    c = s["case"]
    qs, ctx = _lens(c)
    G, o, lse = c["Hq"] // c["Hk"], [], []
    for i, (m, n) in enumerate(zip(qs, ctx)):
        x = q[sum(qs[:i]): sum(qs[:i]) + m].double()
        os_, ls = torch.zeros_like(x), torch.full(x.shape[:2], -math.inf, dtype=torch.float64, device=x.device)
        if n:
            k, v = keys_values(i, n)
            p, j = torch.arange(n - m, n, device=x.device)[:, None], torch.arange(n, device=x.device)
            see = torch.ones((m, n), dtype=torch.bool, device=x.device)
            if c["causal"]:
                see = (j <= p) & ((j > p - c["window"]) if c["window"] else (j >= 0))
            some = see.any(1)
            for h in range(c["Hq"]):
                a = (x[:, h] @ k[h // G].T.contiguous() * s["scale"]).masked_fill(~see, -math.inf)
                ls[:, h] = torch.logsumexp(a, 1)
                os_[some, h] = (torch.softmax(a, 1) @ v[h // G])[some]
        o.append(os_)
        lse.append(ls)
    return [torch.cat(o), torch.cat(lse)]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "heads":
        (q, dq, dwq), (k, dk, dwk) = (_exact_heads(s, s[n], s["w" + n], s["g" + n]) for n in "qk")
        return [q, k, dq, dk, dwq, dwk]
    if c["kind"] == "append" or c["kind"] == "step":
        q, k = (_exact_heads(s, s[n], s["w" + n])[0] for n in "qk")
        v, H = s["v"].double(), torch.ones((1, 1), dtype=torch.float64, device="cuda")
        while H.shape[0] < c["Bv"]:
            H = torch.cat((torch.cat((H, H), 1), torch.cat((H, -H), 1)), 0)
        v = (v.reshape(-1, c["Bv"]) @ H / math.sqrt(c["Bv"])).view(v.shape)
        k, v = _exact_quantized(k), _exact_quantized(v)
        if c["kind"] == "append":
            return [q, k, v]

        def cache(i, n):
            got = _exact_cache(s["pool"], c["Hk"], c["D"], s["table"][i], n)
            got[0][:, n - 1], got[1][:, n - 1] = k[i], v[i]
            return got
        return [q, _exact_attention(s, q, cache)[0]]
    if c["kind"] == "attention":
        return _exact_attention(s, s["q"], lambda i, n: _exact_cache(s["pool"], c["Hk"], c["D"], s["table"][i], n))
    return None                                     # whole numbers: equal to the plain form's or wrong
