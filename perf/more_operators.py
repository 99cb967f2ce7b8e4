"""The operators of attention over streams of tokens, as a serving program calls them.

An attention block rotates its queries and keys by their positions, appends keys
and values to a cache held in 4 bits and attends over it.  The cache's pages
belong to streams, which fork, leave and grow.  Streams advance by prompts,
pieces of long ones, a few drafted tokens, or one token; `granted` says how many
of a call's tokens a stream has.

`run` computes an operator in its plain form, with elementary operations in 32
bits (angles in 64), or where `own` is true calls the framework's layer.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
DEV = "cuda"
BLOCK = 32  # channels that share a scale
TILE = 16   # tokens side by side in a page


def listed():
    return [
        # a layer's queries and keys over four prompts of a large model
        dict(name="rotary prompt bf16", op="rotary", dtype=BF16, batch=4, tokens=4096, heads=32,
             kv_heads=8, head_dim=128, rotary_dim=128, layout="half", scaling="", far=0),
        # generation far into long streams: part of the head, pairs side by side, scaled angles
        dict(name="rotary token f32", op="rotary", dtype=F32, batch=24, tokens=1, heads=12,
             kv_heads=4, head_dim=80, rotary_dim=32, layout="interleaved", scaling="parts",
             far=1000000),
        # keys and values of four prompts into the cache
        dict(name="append prompt bf16", op="append", dtype=BF16, batch=4, tokens=4096, context=0,
             heads=32, kv_heads=8, head_dim=128, page=64, ragged=False),
        # one token for each of 64 streams
        dict(name="append token bf16", op="append", dtype=BF16, batch=64, tokens=1, context=2000,
             heads=32, kv_heads=8, head_dim=128, page=64, ragged=True),
        # four prompts of a large model from their start
        dict(name="attend prompt bf16", op="attend", dtype=BF16, batch=4, tokens=4096, context=0,
             heads=32, kv_heads=8, head_dim=128, page=64, window=0, ragged=False),
        # the next piece of one long document
        dict(name="attend piece bf16", op="attend", dtype=BF16, batch=1, tokens=512,
             context=32768, heads=32, kv_heads=8, head_dim=128, page=64, window=0, ragged=False),
        # sensor streams of unequal lengths that see a bounded past, pages used in a ring
        dict(name="attend window f32", op="attend", dtype=F32, batch=16, tokens=45, context=1500,
             heads=6, kv_heads=2, head_dim=40, page=16, window=250, ragged=True),
        # generation: one token for each of 64 long streams, bound by the cache
        dict(name="attend token bf16", op="attend", dtype=BF16, batch=64, tokens=1, context=8191,
             heads=32, kv_heads=8, head_dim=128, page=64, window=0, ragged=False),
        # a few drafted tokens for each of 32 streams of unequal lengths
        dict(name="attend draft bf16", op="attend", dtype=BF16, batch=32, tokens=6, context=2500,
             heads=16, kv_heads=4, head_dim=64, page=32, window=0, ragged=True),
        # one live stream through a small layer: pure call latency
        dict(name="attend token f32", op="attend", dtype=F32, batch=1, tokens=1, context=300,
             heads=4, kv_heads=4, head_dim=64, page=64, window=0, ragged=False),
        # a search step: 64 streams go on as copies of 16 of them, and each takes a token
        dict(name="pages fork", op="pages", kind="fork", batch=64, layers=4, kv_heads=8,
             head_dim=128, page=64, context=2000, sources=16),
        # streams have left a pool: what is in use moves to its low end
        dict(name="pages compact", op="pages", kind="compact", batch=64, layers=2, kv_heads=8,
             head_dim=128, page=64, context=4000, sources=64),
    ]


# ------------------------------------------------------------------ ranges

SCORES = 4 * 32 * 4096 * 4096      # of the largest attention
CACHED = 64 * 8192 * 8 * 128       # values of the largest cache
VALUES = 4 * 4096 * 40 * 128       # of the largest rotation
BYTES = 2 * 64 * 4000 * 8 * 4 * 34  # that streams hold in the largest pool, at most


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _tokens(rng, longest):
    kind = rng.random()
    if kind < 0.35:
        return 1
    return _log(rng, 2, 12) if kind < 0.5 else _log(rng, 13, longest)


def _head(rng):
    if rng.random() < 0.2:
        return 2 * rng.randint(3, 128)
    return rng.choice((32, 40, 64, 64, 64, 80, 96, 128, 128, 128, 160, 192, 256))


def _draw(rng):
    op = rng.choice(("rotary", "append", "attend", "attend", "attend", "pages"))
    dtype = rng.choice((BF16, BF16, F32))
    kv = rng.choice((1, 2, 3, 4, 8, 8))
    heads, dim = kv * rng.choice((1, 2, 3, 4, 4, 5, 8, 16)), _head(rng)
    page = rng.choice((16, 32, 64, 64, 128, 256))
    batch, tokens = _log(rng, 1, 64), _tokens(rng, 8192)
    if op == "rotary":
        part = dim if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2)
        return dict(op=op, dtype=dtype, batch=batch, tokens=tokens, heads=heads, kv_heads=kv,
                    head_dim=dim, rotary_dim=part, layout=rng.choice(("half", "interleaved")),
                    scaling=rng.choice(("", "linear", "base", "parts")) if part > 2 else "",
                    far=rng.choice((0, _log(rng, 10, 4000000))))
    if op == "pages":
        return dict(op=op, kind=rng.choice(("fork", "compact")), batch=_log(rng, 2, 128),
                    layers=_log(rng, 1, 16), kv_heads=kv, head_dim=dim, page=page,
                    context=_log(rng, 20, 8000), sources=_log(rng, 1, 64))
    context = rng.choice((0, _log(rng, 1, 300), _log(rng, 100, 40000)))
    c = dict(op=op, dtype=dtype, batch=batch, tokens=tokens, context=context, heads=heads,
             kv_heads=kv, head_dim=dim, page=page, ragged=rng.random() < 0.5)
    if op == "attend":
        c["window"] = 0 if rng.random() < 0.6 else _log(rng, 4, 4096)
    return c


def _fits(c):
    if c["op"] == "rotary":
        n = c["batch"] * c["tokens"] * (c["heads"] + c["kv_heads"]) * c["head_dim"]
        return n * (2 if c["dtype"] == F32 else 1) <= VALUES
    if c["op"] == "pages":
        n = c["batch"] * c["layers"] * c["context"] * c["kv_heads"] * _blocks(c) * 34
        return c["sources"] <= c["batch"] and n <= BYTES
    if c["op"] == "append":
        n = c["batch"] * c["tokens"] * c["kv_heads"] * c["head_dim"]
        return n <= VALUES // 5 and c["batch"] * c["context"] * c["kv_heads"] * c["head_dim"] <= CACHED
    held = _stream_pages(c) * c["page"]
    deep = c["batch"] * c["heads"] * c["tokens"] * held * max(1, c["head_dim"] / 128)
    return (deep * (8 if c["dtype"] == F32 else 1) <= SCORES
            and c["batch"] * held * c["kv_heads"] * c["head_dim"] <= CACHED)


def draw(rng):
    while True:
        c = _draw(rng)
        if _fits(c):
            return c


# ------------------------------------------------------------------ a cache's bytes


def _blocks(c):
    return -(-c["head_dim"] // BLOCK)


def _stream_pages(c):
    """Entries of a stream's row of the page table."""
    seen = c["context"] + c["tokens"]
    if c.get("window"):  # the row is a ring: the oldest token's window and the call's tokens
        seen = min(seen, c["window"] + c["tokens"] + c["page"])
    return -(-seen // c["page"]) + 1


def _encode(x):
    """x (..., D) -> codes (..., blocks, 16) of two values a byte and exponents (..., blocks), uint8."""
    D = x.shape[-1]
    nb = -(-D // BLOCK)
    x = torch.nn.functional.pad(x.float(), (0, nb * BLOCK - D)).unflatten(-1, (nb, BLOCK))
    m, e = torch.frexp(x.abs().amax(-1))               # the largest is m 2^e, m in [0.5, 1)
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(-120, 125)
    e = torch.where(m == 0, -120, e)
    v = torch.ldexp(x, -e[..., None])
    a = v.abs()
    # the middles between 0 0.5 1 1.5 2 3 4 6: one that is met goes to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5))
    code = code + 8 * torch.signbit(v).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def _decode(codes, exponents, D):
    """The float32 values (..., D) that codes and exponents stand for."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    steps = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=c.device)
    v = torch.cat((steps, -steps))[c.int()]
    return torch.ldexp(v, exponents[..., None].int() - 127).flatten(-2)[..., :D]


def _views(pool, c):
    """Codes (pages, heads, 2, page, blocks, 16) and exponents (pages, heads, 2, page, blocks) of
    keys and values, by token, in pool (pages, bytes): views of it."""
    P, nb, H = c["page"], _blocks(c), c["kv_heads"]
    heads = pool.view(-1, H, P * nb * 34)
    codes = heads[:, :, :P * nb * 32].unflatten(2, (2, P // TILE, nb, TILE, 16))
    ex = heads[:, :, P * nb * 32:].unflatten(2, (2, P // TILE, nb, TILE))
    return codes.transpose(4, 5), ex.transpose(4, 5)   # (.., tile, token, block, ..)


def _held(s):
    """What the streams hold: (B, entries * page) positions, and the values of keys and values
    (B, heads, entries * page, D) there."""
    c = s["case"]
    P, W, table = c["page"], s["table"].shape[1], s["table"]
    oldest = (s["first"] // P)[:, None]
    at = oldest + (torch.arange(W, device=DEV) - oldest) % W      # which page a slot is of
    pos = at[:, :, None] * P + torch.arange(P, device=DEV)
    pos = torch.where(table[:, :, None] >= 0, pos, 1 << 40).flatten(1)
    codes, ex = _views(s["pool"], c)
    page = table.clamp(min=0).long()
    kv = _decode(codes[page], ex[page], c["head_dim"])            # (B, W, H, 2, tile, token, D)
    kv = kv.permute(3, 0, 2, 1, 4, 5, 6).flatten(3, 5)
    return pos, kv[0], kv[1]


# ------------------------------------------------------------------ inputs


def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _counts(g, c, most, none):
    """How many tokens each stream has: all, or some of them, `none` of them in one."""
    n = torch.full((c["batch"],), most, device=DEV)
    if c["ragged"]:
        n = torch.randint(0, most + 1, (c["batch"],), generator=g, device=DEV)
        n[0] = most
        n[none:none + 1] = 0
    return n.int()


def _projection(g, c):
    """Queries, keys and values side by side, as a projection writes them."""
    B, T, H, K, D = (c[k] for k in ("batch", "tokens", "heads", "kv_heads", "head_dim"))
    u = _normal(g, B, T, H + 2 * K, D).to(DTYPE[c["dtype"]])
    return u.split((H, K, K), 2)


def _keys_like(g, c, *shape):
    """Keys and values as caches hold them: a few channels are larger than the others."""
    wide = torch.exp(_normal(g, c["kv_heads"], 1, c["head_dim"]) * 0.5)
    return _normal(g, *shape) * wide


def _table(g, c, first, tokens, W, pages):
    """Pages of the streams in any order, at their slots of each stream's ring."""
    B, P = c["batch"], c["page"]
    slots = torch.arange(W, device=DEV)
    oldest = (first // P)[:, None]
    at = oldest + (slots - oldest) % W
    table = torch.randperm(pages, generator=g, device=DEV)[:B * W].view(B, W)
    return torch.where(at * P < tokens[:, None], table, -1).int()


def _prepare_attend(g, c):
    B, P, W = c["batch"], c["page"], _stream_pages(c)
    base, granted = _counts(g, c, c["context"], 1), _counts(g, c, c["tokens"], 2)
    tokens = base + granted
    first = torch.zeros_like(base)
    if c.get("window"):
        first = ((base + 1 - c["window"]).clamp(min=0) // P * P).int()
    pages = B * W + 3
    s = dict(case=c, base=base, granted=granted, tokens=tokens, first=first,
             table=_table(g, c, first, tokens, W, pages),
             pool=torch.zeros(pages, c["kv_heads"] * P * _blocks(c) * 34, dtype=torch.uint8,
                              device=DEV))
    s["q"], s["k"], s["v"] = _projection(g, c)
    if c["op"] == "attend":
        codes, ex = _views(s["pool"], c)
        for which in (0, 1):  # of every page, so that what is not held is something else's
            x = _keys_like(g, c, pages, c["kv_heads"], P, c["head_dim"]).to(DTYPE[c["dtype"]])
            cx, xx = _encode(x)
            codes[:, :, which], ex[:, :, which] = (t.unflatten(2, (-1, TILE)) for t in (cx, xx))
    s["refs"] = torch.bincount(s["table"][s["table"] >= 0].long(), minlength=pages).int()
    return s


def _prepare_rotary(g, c):
    s = dict(case=c)
    s["q"], s["k"], _ = _projection(g, c)
    s["positions"] = (torch.randint(0, c["far"] + 1, (c["batch"],), generator=g, device=DEV).int()
                      if c["far"] else torch.zeros(c["batch"], dtype=torch.int32, device=DEV))
    return s


def _prepare_pages(g, c):
    B, P = c["batch"], c["page"]
    W = -(-c["context"] // P) + 2
    tokens = torch.randint(1, c["context"] + 1, (B,), generator=g, device=DEV).int()
    first = torch.zeros_like(tokens)
    pages = B * (W + 2) if c["kind"] == "fork" else 2 * B * W
    s = dict(case=c, tokens=tokens, first=first, table=_table(g, c, first, tokens, W, pages),
             base=tokens.clone(), granted=torch.zeros_like(tokens),
             pool=torch.randint(0, 256, (c["layers"], pages, c["kv_heads"] * P * _blocks(c) * 34),
                                generator=g, device=DEV, dtype=torch.uint8))
    s["refs"] = torch.bincount(s["table"][s["table"] >= 0].long(), minlength=pages).int()
    if c["kind"] == "fork":  # as copies of some of the streams
        s["source"] = torch.randint(0, c["sources"], (B,), generator=g, device=DEV).int()
    else:
        s["left"] = s["table"].clone(), s["refs"].clone()
    return s


def prepare(case, seed):
    g = _generator(seed)
    return {"rotary": _prepare_rotary, "append": _prepare_attend, "attend": _prepare_attend,
            "pages": _prepare_pages}[case["op"]](g, case)


# ------------------------------------------------------------------ plain forms

BASE, FACTOR, ORIGINAL, LOW, HIGH = 10000.0, 8.0, 4096, 1.0, 32.0


def _magnitude(c):
    return 0.1 * math.log(FACTOR) + 1 if c["scaling"] == "parts" else 1.0


def _frequencies(c):
    """Radians a position of each pair, 64 bits."""
    R, base = c["rotary_dim"], BASE
    if c["scaling"] == "base":
        base = base * FACTOR ** (R / (R - 2))
    f = base ** (-torch.arange(0, R, 2, device=DEV, dtype=torch.float64) / R)
    if c["scaling"] == "linear":
        f = f / FACTOR
    if c["scaling"] == "parts":
        keep = ((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f * keep + f / FACTOR * (1 - keep)
    return f


def _plain_rotary(s):
    c = s["case"]
    R, T = c["rotary_dim"], c["tokens"]
    pos = s["positions"][:, None].double() + torch.arange(T, device=DEV)
    angle = pos[:, :, None, None] * _frequencies(c)               # far ones need 64 bits
    cos, sin = ((t * _magnitude(c)).float() for t in (angle.cos(), angle.sin()))

    def turn(x):
        y = x.float()
        if c["layout"] == "half":
            u, w = y[..., :R // 2], y[..., R // 2:R]
            y = torch.cat((u * cos - w * sin, w * cos + u * sin, y[..., R:]), -1)
        else:
            u, w = y[..., 0:R:2], y[..., 1:R:2]
            y = torch.cat((torch.stack((u * cos - w * sin, w * cos + u * sin), -1).flatten(-2),
                           y[..., R:]), -1)
        return y.to(x.dtype)

    return turn(s["q"]), turn(s["k"])


def _places(s):
    """Where the call's tokens lie in the pool: pages (B, T), places in them (B, T), and whether
    the stream has the token."""
    P, W = s["case"]["page"], s["table"].shape[1]
    t = torch.arange(s["case"]["tokens"], device=DEV)
    pos = (s["base"][:, None] + t).long()
    ok = t < s["granted"][:, None]
    return s["table"].gather(1, pos // P % W).long(), pos % P, ok


def _plain_append(s):
    """Encodes the tokens, writes them to the pool, and reads from there what they now stand for."""
    c = s["case"]
    page, at, ok = _places(s)
    codes, ex = _views(s["pool"], c)
    new, got = torch.where(ok), []
    page, at = page[new], at[new]
    for which, x in enumerate((s["k"], s["v"])):
        cx, xx = _encode(x[new])
        codes[page, :, which, at // TILE, at % TILE] = cx
        ex[page, :, which, at // TILE, at % TILE] = xx
        v = _decode(codes[page, :, which, at // TILE, at % TILE],
                    ex[page, :, which, at // TILE, at % TILE], c["head_dim"])
        got.append(torch.zeros_like(x, memory_format=torch.contiguous_format))
        got[-1][new] = v.to(x.dtype)
    return tuple(got)


def _plain_attend(s):
    c = s["case"]
    B, T, H, D = s["q"].shape
    K = c["kv_heads"]
    pos, k, v = _held(s)                                          # (B, L), (B, K, L, D)
    mine = s["base"][:, None] + torch.arange(T, device=DEV)       # (B, T)
    ok = torch.arange(T, device=DEV) < s["granted"][:, None]
    see = (pos[:, None] <= mine[:, :, None]) & ok[:, :, None]
    see &= pos[:, None] >= s["first"][:, None, None]
    if c["window"]:
        see &= pos[:, None] > mine[:, :, None] - c["window"]
    q = s["q"].float().view(B, T, K, H // K, D).permute(0, 2, 3, 1, 4).reshape(B, K, -1, D)
    w = (q @ k.transpose(-1, -2)) * D ** -0.5
    w = w.view(B, K, H // K, T, -1).masked_fill(~see[:, None, None], -math.inf)
    w = torch.exp(w - w.amax(-1, keepdim=True).clamp(min=-1e30))
    w = w / w.sum(-1, keepdim=True).clamp(min=1e-30)
    y = w.view(B, K, -1, w.shape[-1]) @ v
    y = y.view(B, K, H // K, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, H, D)
    return y.to(s["q"].dtype)


def _count(table, pages):
    """How many streams hold each page."""
    n = torch.zeros(pages + 1, dtype=torch.int32, device=DEV)
    at = torch.where(table >= 0, table, pages).flatten().long()
    return n.index_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:pages]


def _plain_fork(s):
    c = s["case"]
    P, W, pages = c["page"], s["table"].shape[1], s["refs"].shape[0]
    src = s["source"].long()
    table, tokens, first = (s[k][src] for k in ("table", "tokens", "first"))
    refs = _count(table, pages)
    # a page for one more token: one that others hold too is copied
    slot = (tokens // P % W).long()[:, None]
    old = table.gather(1, slot)[:, 0].long()
    need = (old < 0) | (refs[old.clamp(min=0)] > 1)
    free = torch.sort((refs > 0).int(), stable=True).indices      # the free ones, lowest first
    new = torch.where(need, free[(torch.cumsum(need, 0) - 1).clamp(min=0)], old)
    table.scatter_(1, slot, new[:, None].int())
    # tiles of tokens that the stream holds
    kept = tokens % P
    tiles = (kept + TILE - 1) // TILE
    pool = s["pool"].view(-1, pages, c["kv_heads"], P * _blocks(c) * 34)
    here = torch.where(need & (kept > 0))[0]
    mask = torch.arange(P // TILE, device=DEV) < tiles[here][:, None]
    n = P * _blocks(c) * 32
    for part, last in ((pool[..., :n], 256), (pool[..., n:], 16)):
        part = part.unflatten(-1, (2, P // TILE, _blocks(c) * last))
        a, b = old[here], new[here]
        part[:, b] = torch.where(mask[:, None, None, :, None], part[:, a], part[:, b])
    # the token is given up again: a page without any other is free again
    table.scatter_(1, slot, torch.where(kept > 0, new, -1)[:, None].int())
    s["table"].copy_(table), s["tokens"].copy_(tokens), s["first"].copy_(first)
    s["refs"].copy_(_count(table, pages))
    return s["table"], s["tokens"], s["refs"], s["pool"]


def _plain_compact(s):
    table, refs = s["left"]
    used = refs > 0
    U = int(used.sum())
    to, at = torch.where(~used[:U])[0], torch.where(used[U:])[0] + U
    s["pool"][:, to] = s["pool"][:, at]
    name = torch.arange(refs.shape[0], device=DEV, dtype=torch.int32)
    name[at] = to.int()
    s["table"].copy_(torch.where(table >= 0, name[table.clamp(min=0).long()], -1))
    s["refs"].copy_(_count(s["table"], refs.shape[0]))
    return s["table"], s["refs"], s["pool"]


def _plain(s):
    op = s["case"]["op"]
    if op == "pages":
        return _plain_fork(s) if s["case"]["kind"] == "fork" else _plain_compact(s)
    return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend}[op](s)


# ------------------------------------------------------------------ the framework's layers


def _layer(s):
    """The layer that a program makes once and keeps, with the pages and their tables."""
    from paper_2204_03418_amd import coinf

    c = s["case"]
    if c["op"] == "rotary":
        scaling = {"": None, "linear": dict(kind="linear", factor=FACTOR),
                   "base": dict(kind="base", factor=FACTOR),
                   "parts": dict(kind="parts", factor=FACTOR, original=ORIGINAL, low=LOW,
                                 high=HIGH)}[c["scaling"]]
        return coinf.CoRotary(c["head_dim"], rotary_dim=c["rotary_dim"], base=BASE,
                              layout=c["layout"], scaling=scaling, magnitude=_magnitude(c),
                              device=DEV)
    state = {k: s[k] for k in ("pool", "table", "tokens", "first", "refs", "base", "granted")}
    state["pool"] = s["pool"].view(c.get("layers", 1), s["refs"].shape[0], -1)
    pages = coinf.CoPages(batch=c["batch"], pages=s["refs"].shape[0], page_tokens=c["page"],
                          stream_pages=s["table"].shape[1], layers=c.get("layers", 1),
                          kv_heads=c["kv_heads"], head_dim=c["head_dim"], state=state)
    if c["op"] == "pages":
        return pages
    return coinf.CoAttention(pages, heads=c["heads"], window=c.get("window") or None,
                             dtype=DTYPE[c["dtype"]])


def _own(s):
    layer = s.get("layer")
    if layer is None:
        layer = s["layer"] = _layer(s)
    c = s["case"]
    if c["op"] == "rotary":
        return layer.forward(s["q"], s["k"], positions=s["positions"])
    if c["op"] == "append":
        layer.append(s["k"], s["v"])
        return layer.read(s["base"], c["tokens"])
    if c["op"] == "attend":
        return layer.attend(s["q"])
    if c["kind"] == "fork":
        layer.select(s["source"])
        layer.reserve(1)
        layer.truncate(layer.base)
        return s["table"], s["tokens"], s["refs"], s["pool"]
    s["table"].copy_(s["left"][0])  # as the streams that left left them
    s["refs"].copy_(s["left"][1])
    layer.compact()
    return s["table"], s["refs"], s["pool"]


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass needs


def work(case):
    c = case
    token = c["kv_heads"] * _blocks(c) * 34  # bytes of a token in the cache
    if c["op"] == "pages":
        if c["kind"] == "fork":  # half a page of each stream
            return dict(bytes=2 * c["batch"] * c["layers"] * c["page"] // 2 * token, flops=0)
        held = c["batch"] * c["context"] // 2   # of a quarter of the pool's pages: three quarters move
        return dict(bytes=2 * c["layers"] * held * 3 // 4 * token, flops=0)
    es = 2 if c["dtype"] == BF16 else 4
    B, T, H, K, D = (c[k] for k in ("batch", "tokens", "heads", "kv_heads", "head_dim"))
    if c["op"] == "rotary":
        n = B * T * (H + K)
        return dict(bytes=2 * es * n * D, flops=3 * n * c["rotary_dim"])
    n = T * (0.5 if c["ragged"] else 1)
    if c["op"] == "append":  # written, read, and their values written
        return dict(bytes=B * n * (2 * token + 4 * es * K * D), flops=B * n * K * D * 8)
    held = c["context"] * (0.5 if c["ragged"] else 1)
    keys = held + (n + 1) / 2
    seen = held + n
    if c["window"]:
        keys, seen = min(keys, c["window"]), min(seen, c["window"] + n)
    return dict(bytes=B * (2 * es * n * H * D + seen * token), flops=4 * B * n * H * D * keys)


# ------------------------------------------------------------------ 64 bits


def _exact_rotary(c, s):
    R, T = c["rotary_dim"], c["tokens"]
    out = []
    for x in (s["q"], s["k"]):
        y = x.double()
        for i in range(R // 2):
            f = BASE ** (-2 * i / R)
            if c["scaling"] == "linear":
                f /= FACTOR
            elif c["scaling"] == "base":
                f = (BASE * FACTOR ** (R / (R - 2))) ** (-2 * i / R)
            elif c["scaling"] == "parts":
                keep = min(1.0, max(0.0, (ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW)))
                f = (keep + (1 - keep) / FACTOR) * f
            u, w = (i, i + R // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
            a = (s["positions"].double()[:, None] + torch.arange(T, device=DEV).double()) * f
            z = torch.complex(x[..., u].double(), x[..., w].double())
            z = z * torch.polar(torch.full_like(a, _magnitude(c)), a)[:, :, None]
            y[..., u], y[..., w] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_quantised(x):
    """The nearest values of the format, x (tokens, heads, D)."""
    y = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    grid = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], device=DEV).double() / 2
    for lo in range(0, x.shape[-1], BLOCK):
        v = x[..., lo:lo + BLOCK].double()
        top = v.abs().amax(-1, keepdim=True)
        # the least power of two that 7 of are not below the largest
        e = torch.ceil(torch.log2((top / 7).clamp(min=1e-300)) - 1e-9)
        e = torch.where(top > 7 * torch.exp2(e), e + 1, e).clamp(-120, 125)
        v = v / torch.exp2(e)
        far = (v.abs()[..., None] - grid).abs()
        odd = torch.arange(8, device=DEV) % 2     # of two as near, the even one
        pick = (far + odd * 1e-12).argmin(-1)
        y[..., lo:lo + BLOCK] = grid[pick] * torch.sign(v) * torch.exp2(e)
    return y


def exact(case, seed):
    c = case
    if c["op"] == "pages":
        return None
    s = prepare(case, seed)
    if c["op"] == "rotary":
        return _exact_rotary(c, s)
    n = [int(v) for v in s["granted"].cpu()]
    if c["op"] == "append":
        out = []
        for x in (s["k"], s["v"]):
            y = torch.zeros(x.shape, dtype=torch.float64, device=DEV)
            for b in range(c["batch"]):
                y[b, :n[b]] = _exact_quantised(x[b, :n[b]])
            out.append(y)
        return tuple(out)
    B, T, H, D = s["q"].shape
    K, P, W = c["kv_heads"], c["page"], s["table"].shape[1]
    pairs = sum(n[b] * (int(s["base"][b]) + n[b]) for b in range(B)) * H * D
    if pairs > 4e12:
        return None
    codes, ex = _views(s["pool"], c)
    grid = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], device=DEV).double() / 2
    y = torch.zeros(B, T, H, D, dtype=torch.float64, device=DEV)
    for b in range(B):
        lo, base, hi = int(s["first"][b]), int(s["base"][b]), int(s["tokens"][b])
        if n[b] == 0:
            continue
        p = torch.arange(lo, hi, device=DEV)
        page, at = s["table"][b, p // P % W].long(), p % P
        kv = []
        for which in (0, 1):
            cd = codes[page, :, which, at // TILE, at % TILE]      # (L, K, blocks, 16)
            sc = torch.exp2(ex[page, :, which, at // TILE, at % TILE].double() - 127)
            x = torch.empty(*cd.shape[:-1], 32, dtype=torch.float64, device=DEV)
            for odd, nib in ((0, cd & 15), (1, cd // 16)):
                x[..., odd::2] = grid[(nib % 8).long()] * (1 - 2 * (nib // 8).double())
            kv.append((x * sc[..., None]).flatten(-2)[..., :D])
        t = torch.arange(base, base + n[b], device=DEV)
        hidden = p > t[:, None]
        if c["window"]:
            hidden |= p <= t[:, None] - c["window"]
        for h in range(H):
            k, v = (x[:, h // (H // K)].contiguous() for x in kv)
            a = s["q"][b, :n[b], h].double() @ k.T.contiguous() / math.sqrt(D)
            a[hidden] = -math.inf
            y[b, :n[b], h] = torch.softmax(a, -1) @ v
    return y
