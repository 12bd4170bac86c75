"""The operators of a drafted-token decode step, as they are measured.

A decoder layer's step around the binary-factorized linears: queries and keys
are rotated to their positions, keys and values are quantised into a paged
cache, the drafted tokens attend to that cache, and at the end the logits of
the drafted tokens are scored. `run` makes one pass through one operator:
with `own` through the library's entry points, otherwise through a plain form
in elementary torch operations (32 bits, rounded once at the end). `exact`
restates each operator in 64 bits.
"""
import math

import torch

DEVICE = torch.device("cuda" if torch.cuda.is_available() else "cpu")

own = False


def _af1():
    import paper_2609_06161_gb300
    return paper_2609_06161_gb300


# -- cases ---------------------------------------------------------------------


def listed():
    return [
        # Eight sequences decode one token each: queries of 32 heads.
        dict(name="rope decode", op="rope", tokens=8, heads=32, dim=128, rot=128, interleaved=False, backward=False,
             dtype="f16", length=8192),
        # The gradient of a prompt's queries, adjacent pairs, half of each head rotated, long positions.
        dict(name="rope prompt backward", op="rope", tokens=2048, heads=32, dim=128, rot=64, interleaved=True,
             backward=True, dtype="f32", length=131072),
        # A decode step's cache write: 16 sequences, one token each, q rotated in the same call.
        dict(name="append decode int8", op="append", kind="int8", batch=16, tokens=1, cached=1000, kv_heads=8, heads=32,
             dim=128, page=64, interleaved=False, dtype="f16", values=False),
        # Four prompts of 2048 tokens written to a 4-bit cache, with the stored values back for the prompt's attention.
        dict(name="append prompt int4", op="append", kind="int4", batch=4, tokens=2048, cached=0, kv_heads=8, heads=0,
             dim=128, page=64, interleaved=False, dtype="f16", values=True),
        # One short sequence read back from an 8-bit cache.
        dict(name="read short e4m3", op="read", kind="e4m3", batch=1, length=777, kv_heads=8, dim=128, page=16),
        # A batch's cache read back, 4 bits, small heads, ragged lengths.
        dict(name="read batch int4", op="read", kind="int4", batch=16, length=8190, kv_heads=8, dim=64, page=128),
        # One sequence, one token, a short cache in 16 bits: the latency of a chat's first tokens.
        dict(name="attend one token f16", op="attend", kind="f16", batch=1, tree=1, length=1000, kv_heads=8, group=4,
             dim=128, page=64, ragged=False),
        # A serving batch: 32 sequences of up to 8192 tokens, one new token each.
        dict(name="attend batch int8", op="attend", kind="int8", batch=32, tree=1, length=8192, kv_heads=8, group=4,
             dim=128, page=64, ragged=False),
        # Four sequences verify trees of up to 16 drafted tokens over small pages.
        dict(name="attend tree 16 e4m3", op="attend", kind="e4m3", batch=4, tree=16, length=6001, kv_heads=8, group=4,
             dim=128, page=16, ragged=True),
        # One long context, 64 drafted tokens, eight queries to a cached head.
        dict(name="attend tree 64 int4", op="attend", kind="int4", batch=1, tree=64, length=32768, kv_heads=8, group=8,
             dim=128, page=128, ragged=False),
        # The scores of five drafted tokens of one sequence.
        dict(name="score draft f32", op="score", rows=5, vocab=32000, given=1, top=8, dtype="f32", banned=False),
        # The scores of a batch of trees (or of a text whose perplexity is measured), some tokens banned.
        dict(name="score batch f16", op="score", rows=512, vocab=128001, given=4, top=20, dtype="f16", banned=True),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw(rng):
    op = rng.choice(("rope", "append", "read", "attend", "attend", "attend", "score"))
    dim = rng.choice((64, 128))
    page = rng.choice((16, 32, 64, 128, 256))
    kind = rng.choice(("f16", "int8", "e4m3", "int4"))
    if op == "rope":
        return dict(op=op, tokens=_log(rng, 1, 8192), heads=rng.randint(1, 64), dim=dim,
                    rot=rng.choice((dim, dim, dim // 2, 24)), interleaved=rng.random() < 0.5,
                    backward=rng.random() < 0.5, dtype=rng.choice(("f16", "f32")), length=_log(rng, 512, 131072))
    if op == "append":
        return dict(op=op, kind=kind, batch=_log(rng, 1, 64), tokens=_log(rng, 1, 2048), cached=rng.randint(0, 300),
                    kv_heads=rng.randint(1, 8), heads=rng.choice((0, 8, 32, 40)), dim=dim, page=page,
                    interleaved=rng.random() < 0.5, dtype=rng.choice(("f16", "f32")), values=rng.random() < 0.5)
    if op == "read":
        return dict(op=op, kind=kind, batch=_log(rng, 1, 32), length=_log(rng, 1, 16384), kv_heads=rng.randint(1, 8),
                    dim=dim, page=page)
    if op == "attend":
        return dict(op=op, kind=kind, batch=_log(rng, 1, 64), tree=_log(rng, 1, 64), length=_log(rng, 1, 32768),
                    kv_heads=rng.randint(1, 8), group=rng.randint(1, 8), dim=dim, page=page, ragged=rng.random() < 0.5)
    return dict(op=op, rows=_log(rng, 1, 1024), vocab=_log(rng, 1000, 150000), given=rng.randint(1, 8),
                top=rng.randint(0, 32), dtype=rng.choice(("f16", "f32")), banned=rng.random() < 0.5)


def draw(rng):
    # Within the memory of the plain forms and the cost of the largest listed case.
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= 6e8 and w["flops"] <= 6e10:
            return case


# -- what every pass has to move and compute -------------------------------------


def _lens(case):
    """Cached tokens of every sequence: ragged, the first the longest, and in larger batches one empty."""
    n, top = case["batch"], case["length"]
    lens = [max(1, round(top * (0.5 + 0.5 * ((1 - 0.6180339887 * b) % 1.0)))) for b in range(n)]
    lens[0] = top
    if n >= 6:
        lens[3] = 0
    return lens


def _counts(case):
    """Drafted tokens of every sequence's tree."""
    t = case["tree"]
    return [t if b == 0 or not case["ragged"] else max(1, t - (5 * b) % t) for b in range(case["batch"])]


def _vector_bytes(kind, dim):
    """Bytes of one cached key or value of one head, with its scales."""
    return {"f16": 2 * dim, "int8": dim + 4, "e4m3": dim + 4, "int4": dim // 2 + 4 * (dim // 32)}[kind]


def _size(dtype):
    return 2 if dtype == "f16" else 4


def work(case):
    op = case["op"]
    if op == "rope":
        n = case["tokens"] * case["heads"]
        return {"bytes": 2 * n * case["dim"] * _size(case["dtype"]) + case["tokens"] * (4 + 4 * case["rot"]),
                "flops": 3 * n * case["rot"]}
    if op == "append":
        n = case["batch"] * case["tokens"]
        kv = n * case["kv_heads"]
        b = 2 * kv * (case["dim"] * _size(case["dtype"]) + _vector_bytes(case["kind"], case["dim"]))
        b += n * case["heads"] * case["dim"] * (_size(case["dtype"]) + 2) + n * (12 + 4 * case["dim"])
        if case["values"]:
            b += 2 * kv * case["dim"] * 2
        return {"bytes": b, "flops": n * case["dim"] * (3 * case["heads"] + 10 * case["kv_heads"])}
    if op == "read":
        n = sum(_lens(case)) * case["kv_heads"]
        m = case["batch"] * case["length"] * case["kv_heads"]
        return {"bytes": 2 * (n * _vector_bytes(case["kind"], case["dim"]) + m * case["dim"] * 2),
                "flops": 2 * n * case["dim"]}
    if op == "attend":
        d, h, g = case["dim"], case["kv_heads"], case["group"]
        b = f = 0
        for n, t in zip(_lens(case), _counts(case)):
            b += 2 * (n + t) * h * _vector_bytes(case["kind"], d)
            f += 4 * (n + t) * t * h * g * d
        b += case["batch"] * case["tree"] * h * g * d * 4
        return {"bytes": b, "flops": f}
    b = case["rows"] * case["vocab"] * _size(case["dtype"]) + case["rows"] * (8 * case["given"] + 8 * case["top"] + 4)
    return {"bytes": b, "flops": 6 * case["rows"] * case["vocab"]}


# -- inputs ------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _dtype(name):
    return torch.float16 if name == "f16" else torch.float32


def _rope_table(length, rot):
    """cos and sin of every position and frequency, float32 [length, rot / 2, 2], as a program keeps it."""
    freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE) / rot)
    angle = torch.arange(length, dtype=torch.float64, device=DEVICE)[:, None] * freq
    return torch.stack((angle.cos(), angle.sin()), -1).float().contiguous()


def _keys(g, n, heads, dim):
    """Keys as projections give them: a few channels of every head are several times the others."""
    big = 1 + 5 * (torch.rand((1, heads, dim), generator=g, device=DEVICE) < 0.05)
    return _randn(g, n, heads, dim) * big


def _pool(case, slots):
    """Empty buffers of a cache with room for `slots` tokens of every sequence, and the table of its pages, in an
    order of their own."""
    per = -(-slots // case["page"])
    pages = per * case["batch"]
    lead = (pages, case["kv_heads"], case["page"])
    d = case["dim"]
    made = {"k_scale": None, "v_scale": None}
    for x in "kv":
        if case["kind"] == "f16":
            made[x] = torch.zeros(lead + (d,), dtype=torch.float16, device=DEVICE)
        elif case["kind"] == "int4":
            made[x] = torch.zeros(lead + (d // 2,), dtype=torch.uint8, device=DEVICE)
            made[x + "_scale"] = torch.zeros(lead + (d // 32, 2), dtype=torch.float16, device=DEVICE)
        else:
            made[x] = torch.zeros(lead + (d,), device=DEVICE,
                                  dtype=torch.int8 if case["kind"] == "int8" else torch.float8_e4m3fn)
            made[x + "_scale"] = torch.zeros(lead, dtype=torch.float32, device=DEVICE)
    return made, per


def _filled(case, g, slots):
    """A cache that holds random keys and values in every slot of every page."""
    made, per = _pool(case, slots)
    table = torch.randperm(per * case["batch"], generator=g, device=DEVICE).view(case["batch"], per).to(torch.int32)
    n = per * case["batch"] * case["page"]
    for x in "kv":
        for at in range(0, n, 1 << 16):  # a part at a time: the caches are large
            m = min(1 << 16, n - at)
            y = _keys(g, m, case["kv_heads"], case["dim"]) if x == "k" else _randn(g, m, case["kv_heads"], case["dim"])
            codes, scale = _quantise(y.half().float(), case["kind"])
            page = torch.arange(at, at + m, device=DEVICE)
            _store(made[x], codes, page // case["page"], page % case["page"])
            if scale is not None:
                _store(made[x + "_scale"], scale, page // case["page"], page % case["page"])
    made["table"] = table
    return made


def _tree_words(parents):
    """Bit j of node i's words: node j is node i or an ancestor of it. Nodes come after their parents."""
    words = []
    for p in range(len(parents)):
        words.append((1 << p) | (words[parents[p]] if parents[p] >= 0 else 0))
    return words


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"case": case}
    if op == "rope":
        s["x"] = _randn(g, case["tokens"], case["heads"], case["dim"]).to(_dtype(case["dtype"]))
        s["positions"] = torch.randint(0, case["length"], (case["tokens"],), generator=g, device=DEVICE,
                                       dtype=torch.int32)
        s["table"] = _rope_table(case["length"], case["rot"])
        s["out"] = torch.empty_like(s["x"])
    elif op == "append":
        b, t = case["batch"], case["tokens"]
        made, per = _pool(case, case["cached"] + t)
        s.update(made)
        s["table"] = torch.randperm(per * b, generator=g, device=DEVICE).view(b, per).to(torch.int32)
        n, dt = b * t, _dtype(case["dtype"])
        s["new_k"] = _keys(g, n, case["kv_heads"], case["dim"]).to(dt)
        s["new_v"] = _randn(g, n, case["kv_heads"], case["dim"]).to(dt)
        s["seq"] = torch.arange(b, device=DEVICE, dtype=torch.int32).repeat_interleave(t)
        s["slot"] = (case["cached"] + torch.arange(t, device=DEVICE, dtype=torch.int32)).repeat(b)
        s["rope"] = _rope_table(case["cached"] + t, case["dim"])
        s["q"] = s["q_out"] = s["k_out"] = s["v_out"] = None
        if case["heads"]:
            s["q"] = _randn(g, n, case["heads"], case["dim"]).to(dt)
            s["q_out"] = torch.empty(s["q"].shape, dtype=torch.float16, device=DEVICE)
        if case["values"]:
            s["k_out"] = torch.empty(s["new_k"].shape, dtype=torch.float16, device=DEVICE)
            s["v_out"] = torch.empty(s["new_v"].shape, dtype=torch.float16, device=DEVICE)
    elif op == "read":
        s.update(_filled(case, g, case["length"]))
        s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEVICE)
        shape = (case["batch"], case["length"], case["kv_heads"], case["dim"])
        s["k_out"] = torch.empty(shape, dtype=torch.float16, device=DEVICE)
        s["v_out"] = torch.empty(shape, dtype=torch.float16, device=DEVICE)
    elif op == "attend":
        t = case["tree"]
        s.update(_filled(case, g, case["length"] + t))
        s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEVICE)
        s["counts"] = torch.tensor(_counts(case), dtype=torch.int32, device=DEVICE) if case["ragged"] else None
        up = torch.rand((case["batch"], t), generator=torch.Generator().manual_seed(seed)).tolist()
        words = []
        for row in up:  # every node hangs under one of the eight before it, or is a root
            words.append(_tree_words([int(i - 1 - u * min(i, 8)) if i else -1 for i, u in enumerate(row)]))
        words = [[[w >> (32 * i) & 0xFFFFFFFF for i in range(-(-t // 32))] for w in row] for row in words]
        s["mask"] = torch.tensor(words, dtype=torch.int64).to(torch.int32).to(DEVICE)  # bit patterns
        heads = case["kv_heads"] * case["group"]
        s["q"] = (1.5 * _randn(g, case["batch"], t, heads, case["dim"])).half()
        s["out"] = torch.empty_like(s["q"])
    else:
        x = 2.5 * _randn(g, case["rows"], case["vocab"])
        top = torch.randint(0, case["vocab"], (case["rows"], 3), generator=g, device=DEVICE)
        x.scatter_(1, top, 14 + 2 * _randn(g, case["rows"], 3))  # what the model thinks likely
        s["tokens"] = torch.randint(0, case["vocab"], (case["rows"], case["given"]), generator=g, device=DEVICE)
        s["tokens"][:, 0] = top[:, 0]
        if case["banned"]:
            kept = x.gather(1, s["tokens"])
            x.masked_fill_(torch.rand(x.shape, generator=g, device=DEVICE) < 0.02, -math.inf)
            x.scatter_(1, s["tokens"], kept)
        s["tokens"] = s["tokens"].to(torch.int32)
        s["logits"] = x.to(_dtype(case["dtype"]))
    if own and op in ("append", "read", "attend"):
        s["cache"] = _af1().KVCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if op == "attend":
            s["workspace"] = s["cache"].make_workspace(s["q"], s["table"])
    return s


# -- the plain forms -----------------------------------------------------------------


def _rotate(x, positions, table, interleaved, sign=1.0):
    """float32 x [tokens, heads, dim] rotated by its positions' angles (`sign` -1: back)."""
    rot = 2 * table.shape[1]
    c, s = table[positions.long()].unbind(-1)
    c, s = c[:, None], sign * s[:, None]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    else:
        a, b = x[..., : rot // 2], x[..., rot // 2: rot]
        y = torch.cat((a * c - b * s, b * c + a * s), -1)
    return torch.cat((y, x[..., rot:]), -1)


def _quantise(x, kind):
    """(codes, scales) of float32 vectors x [..., dim] as a cache of this kind holds them."""
    if kind == "f16":
        return x.half(), None
    if kind == "int4":
        y = x.unflatten(-1, (-1, 32))
        low, high = y.amin(-1), y.amax(-1)
        scale, low = ((high - low) * (1.0 / 15.0)).half(), low.half()
        inv = torch.where(scale > 0, 1.0 / scale.float(), 0.0)
        q = ((y - low.float()[..., None]) * inv[..., None]).round().clamp(0, 15).to(torch.uint8).flatten(-2)
        return q[..., 0::2] | q[..., 1::2] << 4, torch.stack((scale, low), -1)
    top = x.abs().amax(-1)
    scale = top * (1.0 / (127.0 if kind == "int8" else 448.0))
    q = x * torch.where(scale > 0, 1.0 / scale, 0.0)[..., None]
    if kind == "int8":
        return q.round().clamp(-127, 127).to(torch.int8), scale
    return q.clamp(-448, 448).to(torch.float8_e4m3fn), scale


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _store(pool, x, page, row):
    _bytes(pool)[page, :, row] = _bytes(x)


def _values(codes, scale, kind):
    """The float32 vectors that codes and scales stand for."""
    if kind == "f16":
        return codes.float()
    if kind == "int4":
        q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float().unflatten(-1, (-1, 32))
        return (q * scale[..., :1].float() + scale[..., 1:].float()).flatten(-2)
    return codes.float() * scale[..., None]


def _gather(s, x):
    """float32 [batch, slots, kv_heads, dim] of the pages of every sequence."""
    table = s["table"].long()
    scale = s[x + "_scale"]
    codes = _bytes(s[x])[table].view(s[x].dtype)
    y = _values(codes, None if scale is None else scale[table], s["case"]["kind"])
    return y.transpose(2, 3).flatten(1, 2)


def _plain(s):
    case = s["case"]
    op = case["op"]
    if op == "rope":
        y = _rotate(s["x"].float(), s["positions"], s["table"], case["interleaved"], -1.0 if case["backward"] else 1.0)
        return {"out": y.to(s["x"].dtype)}
    if op == "append":
        kind = case["kind"]
        page = s["table"].long()[s["seq"].long(), (s["slot"] // case["page"]).long()]
        row = (s["slot"] % case["page"]).long()
        got = {}
        if s["q"] is not None:
            got["q"] = _rotate(s["q"].float(), s["slot"], s["rope"], case["interleaved"]).half()
        k = _rotate(s["new_k"].float(), s["slot"], s["rope"], case["interleaved"])
        for x, y in (("k", k), ("v", s["new_v"].float())):
            codes, scale = _quantise(y, kind)
            _store(s[x], codes, page, row)
            if scale is not None:
                _store(s[x + "_scale"], scale, page, row)
                got[x + "_scale"] = s[x + "_scale"]
            got[x] = s[x]
            if case["values"]:
                got[x + "_values"] = _values(codes, scale, kind).half()
        return got
    if op == "read":
        here = torch.arange(case["length"], device=DEVICE) < s["lens"][:, None]
        return {x: torch.where(here[..., None, None], _gather(s, x)[:, : case["length"]], 0.0).half() for x in "kv"}
    if op == "attend":
        t, h, d = case["tree"], case["kv_heads"], case["dim"]
        k, v = _gather(s, "k"), _gather(s, "v")
        slot = torch.arange(k.shape[1], device=DEVICE)
        node = slot - s["lens"][:, None]  # [batch, slots]
        index = node.clamp(0, t - 1)
        bit = torch.gather(s["mask"].long(), 2, (index // 32)[:, None].expand(-1, t, -1)) >> (index % 32)[:, None] & 1
        inside = (node >= 0) & (node < t)
        lives = torch.arange(t, device=DEVICE)[None].expand(case["batch"], -1)
        if s["counts"] is not None:
            inside = inside & (node < s["counts"][:, None])
            lives = lives < s["counts"][:, None]
        else:
            lives = lives >= 0
        sees = (node < 0)[:, None] | (inside[:, None] & (bit > 0))  # [batch, tree, slots]
        sees = sees & lives[..., None]
        q = s["q"].float().unflatten(2, (h, -1)).permute(0, 2, 3, 1, 4)  # [batch, kv_heads, group, tree, dim]
        scores = torch.matmul(q, k.permute(0, 2, 3, 1)[:, :, None]) * (1.0 / math.sqrt(d))
        scores = scores.masked_fill(~sees[:, None, None], -math.inf)
        top = scores.amax(-1, keepdim=True)
        p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v.permute(0, 2, 1, 3)[:, :, None]) / torch.where(total > 0, total, 1.0)
        return {"out": o.permute(0, 3, 1, 2, 4).flatten(2, 3).half()}
    x = s["logits"].float()
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    lse = m + z.log()
    got = {"logprobs": torch.gather(x, 1, s["tokens"].long()) - lse,
           "entropy": (z.log() - torch.where(e > 0, e * (x - m), 0.0).sum(-1, keepdim=True) / z)[:, 0]}
    if case["top"]:
        values, ids = torch.sort(x, dim=-1, descending=True, stable=True)
        got["top_logprobs"] = values[:, : case["top"]] - lse
        got["top_ids"] = ids[:, : case["top"]].to(torch.int32)
    return got


def run(s):
    if not own:
        return _plain(s)
    case = s["case"]
    op = case["op"]
    if op == "rope":
        return {"out": _af1().rope(s["x"], s["positions"], s["table"], out=s["out"], interleaved=case["interleaved"],
                                   backward=case["backward"])}
    if op == "append":
        s["cache"].append(s["new_k"], s["new_v"], s["table"], s["seq"], s["slot"], rope=s["rope"], q=s["q"],
                          q_out=s["q_out"], interleaved=case["interleaved"], k_out=s["k_out"], v_out=s["v_out"])
        got = {x: s[x] for x in ("k", "v")}
        got.update({x: s[x] for x in ("k_scale", "v_scale") if s[x] is not None})
        got.update({x: s[y] for x, y in (("q", "q_out"), ("k_values", "k_out"), ("v_values", "v_out"))
                    if s[y] is not None})
        return got
    if op == "read":
        k, v = s["cache"].read(s["table"], s["lens"], count=case["length"], k_out=s["k_out"], v_out=s["v_out"])
        return {"k": k, "v": v}
    if op == "attend":
        return {"out": s["cache"].tree_attention(s["q"], s["table"], s["lens"], mask=s["mask"], counts=s["counts"],
                                                 out=s["out"], workspace=s["workspace"])}
    r = _af1().token_logprobs(s["logits"], s["tokens"], top=case["top"])
    return dict(zip(("logprobs", "entropy", "top_logprobs", "top_ids") if case["top"] else ("logprobs", "entropy"), r))


# -- the definitions in 64 bits ---------------------------------------------------------


def _exact_rotation(x, positions, rope, interleaved, conjugate=False):
    """Pairs as complex numbers times e^(i angle), with the table's cos and sin taken as they are."""
    x = x.double()
    rot = 2 * rope.shape[1]
    turn = torch.view_as_complex(rope.double())[positions.long()][:, None]
    if conjugate:
        turn = turn.conj()
    first = torch.arange(rot // 2, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else rot // 2)
    z = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_values(codes, scale, kind):
    if kind == "int4":
        y = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.float64, device=codes.device)
        y[..., 0::2], y[..., 1::2] = (codes % 16).double(), (codes // 16).double()
        step = scale.double().repeat_interleave(32, dim=-2)
        return y * step[..., 0] + step[..., 1]
    return codes.double() if kind == "f16" else codes.float().double() * scale.double().unsqueeze(-1)


def exact(case, seed):
    s = prepare(case, seed)
    op, kind = case["op"], case.get("kind")
    if op == "rope":
        return {"out": _exact_rotation(s["x"], s["positions"], s["table"], case["interleaved"], case["backward"])}
    if op == "append":
        # Codes are decided by comparisons, so only the scales and the rotated queries have a value in 64 bits.
        got = {x: None for x in ("k", "v")}
        if case["values"]:
            got.update(k_values=None, v_values=None)
        if s["q"] is not None:
            got["q"] = _exact_rotation(s["q"], s["slot"], s["rope"], case["interleaved"])
        k = _exact_rotation(s["new_k"], s["slot"], s["rope"], case["interleaved"])
        for x, y in (("k", k), ("v", s["new_v"].double())):
            if kind == "f16":
                continue
            pool = s[x + "_scale"].double()
            at = s["slot"].long()
            page = s["table"][s["seq"].long(), at // case["page"]].long()
            if kind == "int4":
                y = y.reshape(y.shape[:-1] + (case["dim"] // 32, 32))
                low = y.min(-1).values
                pool[page, :, at % case["page"]] = torch.stack(((y.max(-1).values - low) / 15, low), -1)
            else:
                pool[page, :, at % case["page"]] = y.abs().max(-1).values / (127 if kind == "int8" else 448)
            got[x + "_scale"] = pool
        return got
    if op in ("read", "attend"):
        outs = {"k": [], "v": []}
        found = []
        for b, n in enumerate(_lens(case)):  # a sequence at a time: 64 bits are large
            pages = s["table"][b].long()
            both = {}
            for x in "kv":
                codes = _bytes(s[x])[pages].view(s[x].dtype)
                y = _exact_values(codes, None if kind == "f16" else s[x + "_scale"][pages], kind)
                both[x] = y.permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, case["dim"])
            if op == "read":
                for x in "kv":
                    y = torch.zeros((case["length"], case["kv_heads"], case["dim"]), dtype=torch.float64, device=DEVICE)
                    y[:n] = both[x][:, :n].transpose(0, 1)
                    outs[x].append(y)
                continue
            t = case["tree"]
            live = _counts(case)[b]
            allowed = torch.zeros((t, n + t), dtype=torch.bool)
            allowed[:live, :n] = True
            words = s["mask"][b].cpu().tolist()
            for i in range(live):
                for j in range(live):
                    allowed[i, n + j] = bool(words[i][j // 32] >> (j % 32) & 1)
            allowed = allowed.to(DEVICE)
            o = torch.zeros((t, case["kv_heads"] * case["group"], case["dim"]), dtype=torch.float64, device=DEVICE)
            for h in range(o.shape[1]):
                k, v = (both[x][h // case["group"], : n + t] for x in "kv")
                e = s["q"][b, :, h].double() @ k.T / case["dim"] ** 0.5
                o[:live, h] = torch.softmax(e[:live].masked_fill(~allowed[:live], -math.inf), -1) @ v
            found.append(o)
        return {x: torch.stack(y) for x, y in outs.items()} if op == "read" else {"out": torch.stack(found)}
    got = {"logprobs": [], "entropy": [], "top_logprobs": []}
    for at in range(0, case["rows"], 64):
        lp = torch.log_softmax(s["logits"][at: at + 64].double(), -1)
        got["logprobs"].append(lp.gather(1, s["tokens"][at: at + 64].long()))
        got["entropy"].append(-(lp.exp() * lp.clamp(min=-1e300)).sum(-1))
        got["top_logprobs"].append(lp.topk(case["top"], -1).values)
    got = {x: torch.cat(y) for x, y in got.items()}
    if not case["top"]:
        del got["top_logprobs"]
    else:
        got["top_ids"] = None
    return got
