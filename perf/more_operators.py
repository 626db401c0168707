"""Attention with grouped heads over a paged cache of keys and values, as its speed is measured.

A decoder layer whose heads share keys and values in groups keeps them per token in cache pages.  A step norms and
rotates the new tokens' queries and keys, appends keys and values to the pages, and attends.  Each case is one such
call:

  store    norms of each head, rotation by position, keys and values into their slots, queries for the attention;
  decode   attention of one or a few new tokens per request;
  tree     attention of a tree of drafted tokens: each sees the cached ones and its own ancestors;
  prompt   causal attention of prompts of different lengths, packed one behind the other.

``prepare`` makes what the program holds, ``run`` is the call, ``exact`` the same results in float64.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = torch.device("cuda:0")
EPS = 1e-6


def _store(**kw):
    return dict(dict(op="store", T=32, H=32, G=8, D=128, rope=128, adjacent=False, norm=True, x="bf16", far=100000,
                     layout="token", pad=0, block=64), **kw)


def _attend(op, **kw):
    return dict(dict(op=op, B=1, H=32, G=8, D=128, ctx=1000, new=1, even=True, layout="token", y="bf16", pad=0, block=64),
                **kw)


def listed():
    return [
        # The new tokens of a decode step: launches only.
        _store(name="store-decode-32"),
        # A long prompt's projection, written as the cache wants it.
        _store(name="store-prompt-16381", T=16381, pad=3),
        # Prompts of a model without norms that rotates half of each small head by adjacent pairs; float32 projection.
        _store(name="store-f32-1777", T=1777, H=16, G=2, D=64, rope=32, adjacent=True, norm=False, x="f32", pad=7, block=16,
               layout="head"),
        # One user, an eighth of the heads (eight-way tensor parallel), a short context: latency.
        _attend("decode", name="decode-1", H=8, G=1, ctx=901),
        # A full decode batch of a model with eight queries per key.
        _attend("decode", name="decode-64", B=64, H=64, G=8, ctx=4100, even=False, pad=5, block=16),
        # Long documents, two tokens a step (one drafted), pages by head.
        _attend("decode", name="decode-long-5", B=5, H=32, G=8, ctx=120011, new=2, layout="head"),
        # One user's small tree of drafts.
        _attend("tree", name="tree-1", ctx=2050, new=13),
        # A batch that verifies large trees.
        _attend("tree", name="tree-16", B=16, H=64, G=8, ctx=4000, new=61, even=False, block=32),
        # Short prompts of several users.
        _attend("prompt", name="prompt-short-8", B=8, H=32, G=8, ctx=0, new=700, even=False, block=16),
        # Many very short ones with small heads, float32 results.
        _attend("prompt", name="prompt-packed-61", B=61, H=16, G=4, D=64, ctx=0, new=150, even=False, y="f32", pad=9, block=32),
        # The next part of long prompts, taken in parts.
        _attend("prompt", name="prompt-part-2", B=2, H=32, G=8, ctx=30011, new=259),
        # One long prompt behind a cached prefix.
        _attend("prompt", name="prompt-long-1", B=1, H=32, G=4, ctx=1030, new=7161, block=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("store", "store", "decode", "decode", "tree", "tree", "prompt", "prompt", "prompt"))
    H, D = rng.choice((8, 16, 32, 64)), rng.choice((64, 128, 128))
    common = dict(H=H, G=min(H, rng.choice((1, 2, 4, 8))), D=D, block=rng.choice((16, 32, 64, 128)),
                  layout=rng.choice(("token", "token", "head")), pad=rng.choice((0, 0, 3, 9)))
    G = common["G"]
    if kind == "store":
        return _store(T=_log(rng, 1, 16381 * 48 // max(48, H + 2 * G)), rope=rng.choice((D, D, D // 2, 0)),
                      adjacent=rng.random() < 0.3, norm=rng.random() < 0.7, x=rng.choice(("bf16", "bf16", "f32")),
                      far=_log(rng, 100, 1000000), **common)
    even, y = rng.random() < 0.4, rng.choice(("bf16", "bf16", "f32"))
    if kind == "decode":
        B, new = _log(rng, 1, 96), rng.choice((1, 1, 1, 2, 3))
        return _attend(kind, B=B, ctx=_log(rng, 1, min(120000, 4000000 // (B * G))), new=new, even=even, y=y, **common)
    if kind == "tree":
        B, new = _log(rng, 1, 32), _log(rng, 2, 64)
        return _attend(kind, B=B, ctx=_log(rng, 1, min(60000, 2000000 // (B * G), 250000000 // (B * H * new))), new=new,
                       even=even, y=y, **common)
    B = _log(rng, 1, 61)
    new = _log(rng, 1, int(math.sqrt(1200000000 // (B * H))))
    ctx = rng.choice((0, 0, _log(rng, 1, min(30000, 400000000 // (B * H * new) + 1, 2000000 // (B * G)))))
    return _attend(kind, B=B, ctx=ctx, new=new, even=even, y=y, **common)


# ---------------------------------------------------------------------------
# What a program holds.

def _lengths(c, order):
    """Cached and new tokens of each request: the case's lengths, dealt to the requests in the seed's order."""
    B, rng = c["B"], np.random.default_rng(c["B"] + c["ctx"])
    if c["even"]:
        ctx, new = np.full(B, c["ctx"]), np.full(B, c["new"])
    else:
        ctx = rng.integers(0, c["ctx"] + 1, B)
        new = np.full(B, c["new"]) if c["op"] == "decode" else rng.integers(1, c["new"] + 1, B)
        at = rng.integers(B)
        ctx[at], new[at] = c["ctx"], c["new"]       # one request of the longest kind
    p = order.permutation(B)
    return ctx.astype(np.int64)[p], new.astype(np.int64)[p]


def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV, dtype)


def _cache(pages, c, g):
    """Pages of keys or values, [page][token][head][value]; by head: a head's tokens of a page next to each other."""
    shape = (pages, c["block"], c["G"], c["D"]) if c["layout"] == "token" else (pages, c["G"], c["block"], c["D"])
    t = torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)
    return t if c["layout"] == "token" else t.transpose(1, 2)


def _tree(new, words, rng):
    """Ancestor bits (each token its own too) of trees drafted with a few branches at every node."""
    bits = np.zeros((int(new.sum()), 32 * words), np.uint8)
    at = 0
    for n in new:
        for i in range(n):
            if i:
                bits[at + i] = bits[at + int(rng.integers(max(0, i - 4), i))]
            bits[at + i, i] = 1
        at += n
    return np.packbits(bits, axis=1, bitorder="little").view(np.int32)


def prepare(case, seed):
    c, rng = case, np.random.default_rng(seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    H, G, D = c["H"], c["G"], c["D"]
    s = dict(op=c["op"], H=H, G=G, D=D, block=c["block"])
    if c["op"] == "store":
        T = c["T"] + c["pad"]
        pages = -(-c["T"] // c["block"]) + 3
        slots, position = np.full(T, -1, np.int64), np.full(T, -1, np.int64)
        slots[:c["T"]] = rng.permutation(pages * c["block"])[:c["T"]]
        position[:c["T"]] = (rng.integers(0, c["far"]) + np.arange(c["T"])) % c["far"]
        wide = torch.randn(T, (H + 2 * G) * D, generator=g, device=DEV)
        wide *= torch.exp(0.5 * torch.randn(T, 1, generator=g, device=DEV))
        wide = wide.to(torch.bfloat16) if c["x"] == "bf16" else wide
        q, k, v = (w.view(T, -1, D) for w in wide.split([H * D, G * D, G * D], dim=1))
        weight = lambda: 1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)  # noqa: E731
        rope = c["rope"]
        freq = 10000.0 ** (-np.arange(0, rope, 2, dtype=np.float64) / max(rope, 1))
        return dict(s, q=q, k=k, v=v, q_norm=weight() if c["norm"] else None, k_norm=weight() if c["norm"] else None,
                    freq=_dev(freq, torch.float64) if rope else None, adjacent=c["adjacent"], rope=rope,
                    slots=_dev(slots, torch.int64), position=_dev(position), k_cache=_cache(pages, c, g),
                    v_cache=_cache(pages, c, g))
    ctx, new = _lengths(c, rng)
    seq, T, block = ctx + new, int(new.sum()) + c["pad"], c["block"]
    have = -(-seq // block)
    pages = int(have.sum()) + 1
    table = np.zeros((c["B"], int(have.max())), np.int64)
    table[np.arange(table.shape[1]) < have[:, None]] = rng.permutation(pages)[:pages - 1]
    plan = dict(cu_new=_dev(np.concatenate([[0], np.cumsum(new)])), seq_len=_dev(seq),
                cu_kv=_dev(np.concatenate([[0], np.cumsum(seq)])))
    tree = None
    if c["op"] == "tree":
        words = -(-c["new"] // 32)
        tree = torch.zeros(T, words, dtype=torch.int32, device=DEV)
        tree[:int(new.sum())] = _dev(_tree(new, words, rng))
    q = torch.randn(T, H, D, generator=g, device=DEV) * 1.5       # scores of a spread of 1.5, as trained heads have
    return dict(s, q=q.to(torch.bfloat16), k_cache=_cache(pages, c, g), v_cache=_cache(pages, c, g), table=_dev(table),
                plan=plan, tree=tree, max_new=int(new.max()), max_seq=int(seq.max()), max_kv=int(seq.sum()),
                y=torch.bfloat16 if c["y"] == "bf16" else torch.float32)


# ---------------------------------------------------------------------------
# The calls.

def run(state):
    if own:
        return _own(state)
    return _plain_store(state) if state["op"] == "store" else _plain_attend(state)


def _own(s):
    from paper_2606_29982_amd import caee
    H, G, D = s["H"], s["G"], s["D"]
    T = s["q"].shape[0]
    if s["op"] == "store":
        q = torch.empty(T, H, D, dtype=torch.bfloat16, device=DEV)
        caee.head_store(s["q"], s["k"], s["v"], s["slots"], q, s["k_cache"], s["v_cache"], q_norm=s["q_norm"],
                        k_norm=s["k_norm"], eps=EPS, position=s["position"], freq=s["freq"], adjacent=s["adjacent"])
        return dict(q=q, k_cache=s["k_cache"], v_cache=s["v_cache"])
    if "call" not in s:         # the workspace is kept, as a program keeps it
        att = caee.Heads(heads=H, kv_heads=G, dim=D, scale=D ** -0.5)
        s["call"] = att, caee.alloc_head_workspace(att, T, s["table"].shape[0], s["max_new"], s["max_kv"], DEV,
                                                   tree=s["tree"] is not None)
    att, ws = s["call"]
    y = torch.empty(T, H, D, dtype=s["y"], device=DEV)
    return caee.head_attention(att, s["q"], s["k_cache"], s["v_cache"], s["table"], s["plan"], y, ws,
                               max_new=s["max_new"], max_kv=s["max_kv"], tree=s["tree"])


def _plain_norm(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w


def _plain_rotate(x, s):
    if not s["rope"]:
        return x
    angle = s["position"].double()[:, None, None] * s["freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    r = x[..., :s["rope"]]
    a, b = (r[..., 0::2], r[..., 1::2]) if s["adjacent"] else r.chunk(2, -1)
    pair = (a * cos - b * sin, a * sin + b * cos)
    r = torch.stack(pair, -1).flatten(-2) if s["adjacent"] else torch.cat(pair, -1)
    return torch.cat([r, x[..., s["rope"]:]], -1)


def _plain_store(s):
    q = _plain_rotate(_plain_norm(s["q"], s["q_norm"]), s).to(torch.bfloat16)
    k = _plain_rotate(_plain_norm(s["k"], s["k_norm"]), s).to(torch.bfloat16)
    live = s["slots"] >= 0
    slot = s["slots"][live]
    page, row = slot // s["block"], slot % s["block"]
    s["k_cache"][page, row] = k[live]
    s["v_cache"][page, row] = s["v"][live].to(torch.bfloat16)
    return dict(q=q, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_attend(s):
    """All requests at once, padded to the longest: [B, G, H / G * n, D] against [B, G, L, D]."""
    p, block, L, n, H, G, D = s["plan"], s["block"], s["max_seq"], s["max_new"], s["H"], s["G"], s["D"]
    cu, seq = p["cu_new"].long(), p["seq_len"].long()
    B, new = seq.numel(), cu[1:] - cu[:-1]
    j, i = torch.arange(L, device=DEV), torch.arange(n, device=DEV)
    page = s["table"].long()[:, (j // block).clamp(max=s["table"].shape[1] - 1)]
    at = (cu[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().view(B, n, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(B, G, H // G * n, D)
    k = s["k_cache"][page, j % block].float().permute(0, 2, 1, 3)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, G, H // G, n, L)
    del k
    score *= D ** -0.5
    base = (seq - new)[:, None]
    if s["tree"] is None:
        seen = j <= (base + i)[:, :, None]
    else:
        bit = j - base                                                      # [B, L]: number of a new token
        word = s["tree"][at].long().gather(2, (bit // 32).clamp(0, s["tree"].shape[1] - 1)[:, None].expand(B, n, L))
        seen = (bit < 0)[:, None] | ((word >> (bit % 32)[:, None]) & 1).bool()
    seen = seen & (j < seq[:, None])[:, None, :]
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    score.sub_(torch.where(torch.isfinite(top), top, 0.0)).exp_()
    total = score.sum(-1, keepdim=True)
    score.div_(torch.where(total > 0, total, 1.0))
    v = s["v_cache"][page, j % block].float().permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(score.view(B, G, H // G * n, L), v).view(B, G, H // G, n, D)
    y = torch.zeros(s["q"].shape[0], H, D, dtype=s["y"], device=DEV)
    live = i < new[:, None]
    y[at[live]] = o.permute(0, 3, 1, 2, 4).reshape(B, n, H, D)[live].to(s["y"])
    return y


# ---------------------------------------------------------------------------
# What a pass cannot do without.

def work(case):
    c = case
    H, G, D = c["H"], c["G"], c["D"]
    if c["op"] == "store":
        values = c["T"] * (H + 2 * G) * D
        return dict(bytes=values * ((2 if c["x"] == "bf16" else 4) + 2) + 12 * c["T"], flops=7 * c["T"] * (H + G) * D)
    ctx, new = _lengths(c, np.random.default_rng(1))
    T = int(new.sum())
    pairs = float((new * ctx + (new if c["op"] == "tree" else new * (new + 1) // 2)).sum())
    io = T * H * D * (2 + (2 if c["y"] == "bf16" else 4)) + 4 * G * D * int((ctx + new).sum())
    return dict(bytes=int(io), flops=int(4 * pairs * H * D))


# ---------------------------------------------------------------------------
# The definitions in 64 bits.

def _exact_head(x, w, s):
    """[T, heads, D] in float64: norm, then each pair as a complex number turned by its angle."""
    x = x.to(torch.float64)
    if w is not None:
        x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * w.to(torch.float64)
    r = s["rope"]
    if r:
        first, second = (slice(0, r, 2), slice(1, r, 2)) if s["adjacent"] else (slice(0, r // 2), slice(r // 2, r))
        turn = torch.exp(1j * (s["position"].to(torch.float64).view(-1, 1, 1) * s["freq"]))
        z = torch.complex(x[..., first], x[..., second]) * turn
        x = x.clone()
        x[..., first], x[..., second] = z.real, z.imag
    return x


def exact(case, seed):
    s = prepare(case, seed)
    f8 = torch.float64
    H, G, D, block = s["H"], s["G"], s["D"], s["block"]
    if s["op"] == "store":
        q, k = _exact_head(s["q"], s["q_norm"], s), _exact_head(s["k"], s["k_norm"], s)
        kc, vc = s["k_cache"].to(f8), s["v_cache"].to(f8)
        t = torch.nonzero(s["slots"] >= 0)[:, 0]
        where = torch.div(s["slots"][t], block, rounding_mode="floor"), torch.remainder(s["slots"][t], block)
        kc[where], vc[where] = k[t], s["v"].to(f8)[t]
        return dict(q=q, k_cache=kc, v_cache=vc)
    cu, seq = s["plan"]["cu_new"].tolist(), s["plan"]["seq_len"].tolist()
    y = torch.zeros(s["q"].shape[0], H, D, dtype=f8, device=DEV)
    for b, L in enumerate(seq):
        n = cu[b + 1] - cu[b]
        pos = torch.arange(L, device=DEV)
        page, row = s["table"][b, pos // block].long(), pos % block
        hide = torch.zeros(n, L, dtype=torch.bool, device=DEV)
        if s["tree"] is None:
            hide[:, L - n:] = torch.ones(n, n, device=DEV).triu(1).bool()
        else:
            words = s["tree"][cu[b]:cu[b + 1]].cpu().numpy().view(np.uint8)
            hide[:, L - n:] = torch.from_numpy(np.unpackbits(words, axis=1, bitorder="little")[:, :n] == 0).to(DEV)
        for g in range(G):
            k, v = s["k_cache"][page, row, g].to(f8), s["v_cache"][page, row, g].to(f8)
            for h in range(g * (H // G), (g + 1) * (H // G)):
                a = (s["q"][cu[b]:cu[b + 1], h].to(f8) @ k.t()) / math.sqrt(D)
                y[cu[b]:cu[b + 1], h] = torch.softmax(a.masked_fill(hide, -math.inf), 1) @ v
    return y
