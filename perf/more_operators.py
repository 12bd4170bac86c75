"""What follows the logits of drafted tokens, as it is measured.

A step that serves drafted tokens ends so: logits become probabilities
(temperature, the k largest, a least share of the largest), the drafted tokens
are verified against them with given random numbers, the accepted tokens' keys
and values move behind the prefix, and the cache's pages are shared, copied,
reserved and released for the next step. `run` makes one pass through one of
these operators: with `own` through the library's entry points, otherwise
through a plain form in elementary torch operations. `exact` restates what is
computed in 64 bits.
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
        # The tree of one sequence: five rows of logits, one setting for all of them.
        dict(name="probs draft f32", op="probs", rows=5, vocab=32000, dtype="f32", cut="all", top_k=50, banned=False),
        # The trees of a batch, each sequence with its own temperature, k and least share; some tokens banned.
        dict(name="probs batch f16", op="probs", rows=512, vocab=128001, dtype="f16", cut="rows", top_k=200, banned=True),
        # A batch's rows sampled from all of the vocabulary, as a draft model's are.
        dict(name="probs whole f32", op="probs", rows=128, vocab=128000, dtype="f32", cut="none", top_k=0, banned=False),
        # Eight sequences with a chain of five drafted tokens each, drawn from a draft model.
        dict(name="verify chains", op="verify", batch=8, nodes=6, vocab=32000, draft="drawn", chain=True),
        # Trees of a batch whose siblings were drawn without repetition.
        dict(name="verify distinct trees", op="verify", batch=16, nodes=16, vocab=128001, draft="distinct", chain=False),
        # A large batch with trees of guesses (the draft's likeliest tokens), no draft probabilities.
        dict(name="verify guessed trees", op="verify", batch=64, nodes=32, vocab=128000, draft="guessed", chain=False),
        # One sequence accepts a path of its tree: two layers of a small model.
        dict(name="compact chat int8", op="compact", kind="int8", layers=2, batch=1, nodes=16, length=500, kv_heads=2,
             dim=64, page=32),
        # A batch accepts its paths in all layers.
        dict(name="compact batch f16", op="compact", kind="f16", layers=32, batch=64, nodes=32, length=100, kv_heads=8,
             dim=128, page=64),
        # A beam step copies the last pages of a few sequences, in part filled.
        dict(name="copy beams e4m3", op="copy", kind="e4m3", layers=4, copies=4, pages=64, kv_heads=8, dim=128, page=16,
             full=False),
        # Pages copied for many forked sequences in all layers.
        dict(name="copy forks int4", op="copy", kind="int4", layers=16, copies=100, pages=256, kv_heads=8, dim=128,
             page=128, full=True),
        # A beam search of four sequences, four beams each: the table's step.
        dict(name="pages beams", op="pages", batch=16, beams=4, length=300, nodes=1, page=16, pages=1000),
        # The table's step of a large server: 256 sequences, some sharing prompts, up to 64 drafted tokens each.
        dict(name="pages server", op="pages", batch=256, beams=8, length=8000, nodes=64, page=32, pages=131072),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw(rng):
    op = rng.choice(("probs", "probs", "verify", "verify", "compact", "copy", "pages"))
    kind = rng.choice(("f16", "int8", "e4m3", "int4"))
    dim, page = rng.choice((64, 128)), rng.choice((16, 32, 64, 128, 256))
    if op == "probs":
        vocab = _log(rng, 1000, 150000)
        return dict(op=op, rows=_log(rng, 1, 1024), vocab=vocab, dtype=rng.choice(("f16", "f32")),
                    cut=rng.choice(("none", "all", "rows", "rows")), top_k=_log(rng, 1, vocab), banned=rng.random() < 0.5)
    if op == "verify":
        return dict(op=op, batch=_log(rng, 1, 128), nodes=_log(rng, 1, 64), vocab=_log(rng, 1000, 150000),
                    draft=rng.choice(("drawn", "distinct", "guessed")), chain=rng.random() < 0.3)
    if op == "compact":
        return dict(op=op, kind=kind, layers=rng.randint(1, 32 if kind == "f16" else 16), batch=_log(rng, 1, 128),
                    nodes=_log(rng, 1, 64), length=rng.randint(0, 200), kv_heads=rng.randint(1, 8), dim=dim, page=page)
    if op == "copy":
        n = _log(rng, 1, 300)
        return dict(op=op, kind=kind, layers=rng.randint(1, 16), copies=n, pages=2 * n + rng.randint(0, 50),
                    kv_heads=rng.randint(1, 8), dim=dim, page=page, full=rng.random() < 0.5)
    batch, length, nodes = _log(rng, 1, 512), _log(rng, 1, 8000), _log(rng, 1, 64)
    need = batch * (-(-(length + nodes) // page) + 2)
    return dict(op=op, batch=batch, beams=rng.randint(1, 8), length=length, nodes=nodes, page=page,
                pages=need + _log(rng, 1, need))


def _state_bytes(case):
    """Most of what the inputs hold."""
    if case["op"] == "verify":
        return 4 * case["batch"] * case["nodes"] * case["vocab"] * (1 if case["draft"] == "guessed" else 2)
    if case["op"] in ("compact", "copy"):
        pages = case["pages"] if case["op"] == "copy" else case["batch"] * _columns(case)
        return 2 * case["layers"] * pages * case["page"] * case["kv_heads"] * _vector_bytes(case["kind"], case["dim"])
    return 0


def draw(rng):
    # Within the memory of the plain forms and the cost of the largest listed case.
    while True:
        case = _draw(rng)
        w = work(case)
        if w["bytes"] <= 3.8e8 and _state_bytes(case) <= 1e9 and case.get("pages", 0) <= 200000:
            return case


# -- what every pass has to move and compute -------------------------------------


def _columns(case):
    """Pages of a sequence's row of the table."""
    return -(-(case["length"] + case["nodes"]) // case["page"])


def _vector_bytes(kind, dim):
    """Bytes of one cached key or value of one head, with its scales."""
    return {"f16": 2 * dim, "int8": dim + 4, "e4m3": dim + 4, "int4": dim // 2 + 4 * (dim // 32)}[kind]


def _copied_rows(case):
    """Rows of every copied page."""
    return [case["page"] if case["full"] else 1 + (5 * i + 7) % case["page"] for i in range(case["copies"])]


def _mean_moves(case):
    """Tokens of a sequence's accepted path that move: about a quarter of the nodes are on it, the first stays."""
    return max(0, (case["nodes"] + 3) // 4 - 1)


def work(case):
    op = case["op"]
    if op == "probs":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * ((2 if case["dtype"] == "f16" else 4) + 4), "flops": 6 * n}
    if op == "verify":
        # The row of probabilities that the following token is drawn from, the draft's row where it was rejected.
        n = case["batch"] * case["vocab"] * (1 if case["draft"] == "guessed" else 2)
        return {"bytes": 4 * n + 28 * case["batch"] * case["nodes"], "flops": 3 * n}
    if op == "compact":
        rows = case["batch"] * _mean_moves(case) * case["kv_heads"] * case["layers"]
        return {"bytes": 4 * rows * _vector_bytes(case["kind"], case["dim"]) + 8 * case["batch"] * case["nodes"],
                "flops": 0}
    if op == "copy":
        rows = sum(_copied_rows(case)) * case["kv_heads"] * case["layers"]
        return {"bytes": 4 * rows * _vector_bytes(case["kind"], case["dim"]) + 12 * case["copies"], "flops": 0}
    # Counts of the pages, once; the table, once for each of the three calls' look at it; what they change is little.
    return {"bytes": 4 * case["pages"] + 8 * case["batch"] * _columns(case) + 28 * case["batch"], "flops": 0}


# -- inputs ------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device=DEVICE)


def _randint(g, lo, hi, *shape):
    return torch.randint(lo, hi, shape, generator=g, device=DEVICE, dtype=torch.int32)


def _logits(g, rows, vocab):
    """Most entries unlikely, a few that the model thinks likely."""
    x = _randn(g, rows, vocab).mul_(2.5)
    part = vocab // 6  # each in a part of its own: no place is written twice
    top = torch.arange(6, device=DEVICE) * part + torch.randint(0, part, (rows, 6), generator=g, device=DEVICE)
    return x.scatter_(1, top, 11 + 2 * _randn(g, rows, 6))


def _kept_layers(case, g, pages):
    """The layers' caches: codes and scales of random keys and values in every slot."""
    lead, d = (pages, case["kv_heads"], case["page"]), case["dim"]
    layers = []
    for _ in range(case["layers"]):
        made = {"k_scale": None, "v_scale": None}
        for x in "kv":
            if case["kind"] == "f16":
                made[x] = _randn(g, *lead, d).half()
            elif case["kind"] == "int4":
                made[x] = torch.randint(0, 256, lead + (d // 2,), generator=g, device=DEVICE, dtype=torch.uint8)
                made[x + "_scale"] = (0.1 + _rand(g, *lead, d // 32, 2)).half()
            else:
                made[x] = torch.randint(-127, 128, lead + (d,), generator=g, device=DEVICE, dtype=torch.int8)
                if case["kind"] == "e4m3":
                    made[x] = made[x].float().to(torch.float8_e4m3fn)
                made[x + "_scale"] = 0.01 + 0.1 * _rand(g, *lead)
        layers.append(made)
    return layers


def _trees(case, seed):
    """Parents of every node, and its place among its siblings. A node has up to eight children, close
    behind it."""
    n = case["nodes"]
    up = torch.rand((case["batch"], n), generator=torch.Generator().manual_seed(seed)).tolist()
    parents, places = [], []
    for row in up:
        p = [-1 if i == 0 else i - 1 if case["chain"] else int(i - 1 - u * min(i, 7)) for i, u in enumerate(row)]
        parents.append(p)
        places.append([p[:i].count(p[i]) for i in range(n)])
    return [torch.tensor(x, dtype=torch.int32, device=DEVICE) for x in (parents, places)]


def _prepare_verify(case, g, seed):
    b, n, v = case["batch"], case["nodes"], case["vocab"]
    x = _logits(g, b * n, v)
    s = {"probs": torch.softmax(x, -1).view(b, n, v), "draft": None}
    for at in range(0, b * n, 64):  # the draft model is near the target: a part at a time
        x[at: at + 64] += 0.6 * _randn(g, min(64, b * n - at), v)
    q = torch.softmax(x, -1)
    s["parents"], places = _trees(case, seed)
    if case["draft"] == "guessed":
        drawn = torch.topk(x, 8, -1).indices
    else:
        s["draft"] = q.view(b, n, v)
        drawn = torch.multinomial(q, 8, replacement=case["draft"] == "drawn", generator=g)
    up = s["parents"].long().clamp(min=0)
    s["tokens"] = drawn.view(b, n, 8)[torch.arange(b, device=DEVICE)[:, None], up, places.long()].to(torch.int32)
    s["uniforms"] = _rand(g, b, n)
    s["counts"] = _randint(g, 1, n + 1, b)
    s["counts"][0] = n
    return s


def _lens(case):
    """Cached tokens of every sequence: ragged, the first the longest."""
    top = case["length"]
    return [round(top * (0.5 + 0.5 * ((1 - 0.6180339887 * b) % 1.0))) if b else top for b in range(case["batch"])]


def _prepare_pages(case, g):
    """Groups of beams that share their prompt's pages; every sequence has its own pages after that."""
    b, ps, n = case["batch"], case["page"], case["nodes"]
    columns = _columns(case) + 1
    group = [i - i % case["beams"] for i in range(b)]
    lens = [_lens(case)[x] for x in group]
    table, used = [[-1] * columns for _ in range(b)], 0
    for i in range(b):
        held = -(-lens[i] // ps)
        shared = held // 2
        for c in range(held):
            if c < shared and group[i] != i:
                table[i][c] = table[group[i]][c]
            else:
                table[i][c], used = used, used + 1
    table = torch.tensor(table, dtype=torch.int32, device=DEVICE)
    where = torch.randperm(case["pages"], generator=g, device=DEVICE).to(torch.int32)
    table = torch.where(table >= 0, where[table.long().clamp(min=0)], table)
    refs = torch.bincount(table.long().flatten() + 1, minlength=case["pages"] + 1)[1:].to(torch.int32)
    first = torch.arange(b, device=DEVICE, dtype=torch.int32) // case["beams"] * case["beams"]
    size = (torch.tensor(b, device=DEVICE) - first).clamp(max=case["beams"])
    counts = _randint(g, 1, n + 1, b)
    s = {"table": table, "refs": refs, "lens": torch.tensor(lens, dtype=torch.int32, device=DEVICE), "counts": counts,
         "parents": (first + (_rand(g, b) * size).floor()).to(torch.int32)}
    s["kept"] = s["lens"] + (_rand(g, b) * (counts + 1)).floor().to(torch.int32)
    return s


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = {"case": case}
    if op == "probs":
        rows, vocab = case["rows"], case["vocab"]
        x = _logits(g, rows, vocab)
        if case["banned"]:
            top = x.argmax(-1, keepdim=True)
            kept = x.gather(1, top)
            x.masked_fill_(_rand(g, rows, vocab) < 0.02, -math.inf)
            x.scatter_(1, top, kept)
        s["logits"] = x.half() if case["dtype"] == "f16" else x
        s["temperature"], s["top_k"], s["min_p"] = 0.8, 0, 0.0
        if case["cut"] == "all":
            s["top_k"], s["min_p"] = case["top_k"], 0.02
        elif case["cut"] == "rows":  # of every sequence: a few greedy, a few that keep all tokens
            s["temperature"] = torch.where(_rand(g, rows) < 0.1, 0.0, 0.5 + _rand(g, rows))
            s["top_k"] = torch.where(_rand(g, rows) < 0.2, 0, _randint(g, 1, case["top_k"] + 1, rows))
            s["min_p"] = torch.where(_rand(g, rows) < 0.5, 0.0, 0.1 * _rand(g, rows))
        s["out"] = torch.empty((rows, vocab), dtype=torch.float32, device=DEVICE)
    elif op == "verify":
        s.update(_prepare_verify(case, g, seed))
    elif op == "compact":
        b, n, columns = case["batch"], case["nodes"], _columns(case)
        s["layers"] = _kept_layers(case, g, b * columns)
        s["table"] = torch.randperm(b * columns, generator=g, device=DEVICE).view(b, columns).to(torch.int32)
        s["first"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEVICE)
        s["counts"] = torch.full((b,), _mean_moves(case) + 1, dtype=torch.int32, device=DEVICE)
        # The first node, then nodes in ascending order, with no two the same, and -1 behind the path.
        path = torch.sort(_rand(g, b, n - 1).topk(_mean_moves(case), -1).indices + 1, -1).values if n > 1 else \
            torch.zeros((b, 0), dtype=torch.int64, device=DEVICE)
        s["index"] = torch.full((b, n), -1, dtype=torch.int32, device=DEVICE)
        s["index"][:, 0] = 0
        s["index"][:, 1: 1 + path.shape[1]] = path.to(torch.int32)
    elif op == "copy":
        s["layers"] = _kept_layers(case, g, case["pages"])
        n = case["copies"]
        pages = torch.randperm(case["pages"], generator=g, device=DEVICE)[: 2 * n].to(torch.int32)
        rows = torch.tensor(_copied_rows(case), dtype=torch.int32, device=DEVICE)
        s["copies"] = torch.stack((pages[:n], pages[n:], rows), -1).contiguous()
    else:
        s.update(_prepare_pages(case, g))
    if own and op in ("compact", "copy"):
        s["caches"] = [_af1().KVCache(x["k"], x["v"], x["k_scale"], x["v_scale"]) for x in s["layers"]]
    if own and op == "pages":
        s["pages"] = _af1().PageTable(s["table"], s["refs"], case["page"])
    return s


# -- the plain forms -----------------------------------------------------------------


def _column(x, rows, dtype):
    return x.to(dtype)[:, None] if torch.is_tensor(x) else torch.full((rows, 1), x, dtype=dtype, device=DEVICE)


def _plain_probs(s):
    x = s["logits"].float()
    rows, vocab = x.shape
    t = _column(s["temperature"], rows, torch.float32)
    k = _column(s["top_k"], rows, torch.int64)
    p = _column(s["min_p"], rows, torch.float32).double()
    top = x.amax(-1, keepdim=True)
    greedy = t < 1e-30
    # The cut of a least share of the largest, in 64 bits: entries may be next to it.
    keep = x.double() >= top.double() + t.double() * torch.log(p)
    if s["case"]["cut"] != "none":
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices
        rank = torch.empty_like(order).scatter_(1, order, torch.arange(vocab, device=DEVICE).expand(rows, -1))
        keep &= (rank < k) | (k <= 0)
    at = torch.arange(vocab, device=DEVICE)
    first = torch.where(x == top, at, vocab).amin(-1, keepdim=True)
    e = torch.exp((x - top) / torch.where(greedy, 1.0, t))
    e = torch.where(greedy, (at == first).float(), torch.where(keep, e, 0.0))
    return {"probs": e / e.sum(-1, keepdim=True)}


_UNIT = 2.0 ** 40  # masses are whole numbers of its inverse: their sums do not depend on an order


def _mass(r):
    """The masses of probabilities r (float32, 0 to 1), as int64."""
    return torch.round(r.double() * _UNIT).long()


def _plain_verify(s):
    probs, draft, tokens, parents, u = s["probs"], s["draft"], s["tokens"].long(), s["parents"].long(), s["uniforms"]
    b, n, v = probs.shape
    seq = torch.arange(b, device=DEVICE)
    at = torch.zeros(b, dtype=torch.int64, device=DEVICE)
    length = torch.ones(b, dtype=torch.int64, device=DEVICE)
    path = torch.full((b, n + 1), -1, dtype=torch.int64, device=DEVICE)
    path[:, 0] = 0
    one = torch.ones(b, dtype=torch.float64, device=DEVICE)
    c, z, zq = torch.zeros_like(one), one.clone(), one.clone()
    gone = torch.zeros((b, v), dtype=torch.bool, device=DEVICE)  # tokens rejected at this node
    distinct = s["case"]["draft"] == "distinct"
    for i in range(1, n):
        here = (parents[:, i] == at) & (i < s["counts"])
        t = tokens[:, i]
        p = probs[seq, at, t].clamp(0, 1)
        if draft is None:
            r = torch.where(gone[seq, t], 0.0, p).double()
            take = here & (u[:, i].double() * z < r)
            lost = here & ~take
            z = torch.where(lost, z - r, z)
        else:
            q = draft[seq, at, t].clamp(0, 1)
            seen = gone[seq, t]
            here = here & (zq > 0) & ~(seen & distinct)
            r = torch.where(seen, 0.0, (p - c.float() * q).clamp(min=0)).double()
            take = here & (u[:, i].double() * q.double() * z < r * zq)
            lost = here & ~take
            c = torch.where(lost, c + z / zq, c)
            if distinct:
                zq = torch.where(lost, zq - q.double(), zq)
        gone[seq, t] |= lost
        if draft is not None:
            rest = (probs[seq, at] - c.float()[:, None] * draft[seq, at]).clamp(0, 1).masked_fill(gone, 0.0)
            z = torch.where(lost, _mass(rest).sum(-1).double() / _UNIT, z)
        path.scatter_(1, torch.where(take, length, n)[:, None], i)
        length = length + take
        at = torch.where(take, i, at)
        c, z, zq = torch.where(take, 0.0, c), torch.where(take, one, z), torch.where(take, one, zq)
        gone &= ~take[:, None]
    whole = probs[seq, at].clamp(0, 1)
    rest = whole if draft is None else (whole - c.float()[:, None] * draft[seq, at]).clamp(0, 1)
    mass = _mass(rest.masked_fill(gone, 0.0))
    mass = torch.where(mass.sum(-1, keepdim=True) > 0, mass, _mass(whole))
    sums = mass.cumsum(-1)
    bound = torch.floor(u[:, 0].double().clamp(0, 1 - 2.0 ** -24) * sums[:, -1].double()).long()
    following = (sums <= bound[:, None]).sum(-1)
    following = torch.where(sums[:, -1] > 0, following, -1)
    keep = torch.arange(n, device=DEVICE) < length[:, None]
    return {"path": torch.where(keep, path[:, :n], -1).to(torch.int32), "lengths": length.to(torch.int32),
            "following": following.to(torch.int32)}


def _bytes(x):
    return x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x


def _plain_compact(s):
    page = s["case"]["page"]
    n = s["index"].shape[1]
    j = torch.arange(n, device=DEVICE)
    index = torch.where(j < s["counts"][:, None], s["index"].long(), j)
    first = s["first"].long()[:, None]
    source, target = first + index, torch.where(j < s["counts"][:, None], first + j, first + index)
    seq = torch.arange(first.shape[0], device=DEVICE)[:, None]
    table = s["table"].long()
    source_page, target_page = table[seq, source // page], table[seq, target // page]
    for layer in s["layers"]:
        for x in layer.values():
            if x is not None:
                y = _bytes(x)
                y[target_page, :, target % page] = y[source_page, :, source % page]
    return _pools(s)


def _plain_copy(s):
    page = s["case"]["page"]
    source, target, rows = s["copies"].long().unbind(-1)
    inside = torch.arange(page, device=DEVICE) < rows[:, None]
    for layer in s["layers"]:
        for x in layer.values():
            if x is not None:
                y = _bytes(x)
                mask = inside.view(inside.shape[0], 1, page, *(1,) * (y.dim() - 3))
                y[target] = torch.where(mask, y[source], y[target])
    return _pools(s)


def _pools(s):
    return [[x for x in layer.values() if x is not None] for layer in s["layers"]]


def _plain_pages(s):
    table, refs, page = s["table"], s["refs"], s["case"]["page"]
    b, columns = table.shape
    count = refs.shape[0]

    def change(entries, by):  # the counts of entries that hold a page
        refs.scatter_add_(0, entries.long().clamp(min=0).flatten(), torch.where(entries >= 0, by, 0).to(torch.int32).flatten())

    # Every sequence goes on from its parent.
    moved = torch.where(s["parents"][:, None] >= 0, table[s["parents"].long().clamp(min=0)], -1)
    change(moved, 1)
    change(table, -1)
    table.copy_(moved)

    # Pages of their own for the slots to come: where there is none, and where others hold it too but for the last.
    first, last = s["lens"][:, None] // page, (s["lens"] + s["counts"] - 1)[:, None] // page
    at = torch.arange(columns, device=DEVICE)
    inside = (at >= first) & (at <= last) & (s["counts"] > 0)[:, None]
    held, index = table >= 0, table.long().clamp(min=0)
    shared = inside & held & (refs[index] > 1)
    order = torch.arange(b * columns, device=DEVICE).view(b, columns)
    writers = torch.zeros(count, dtype=torch.int32, device=DEVICE)
    writers.scatter_add_(0, index.flatten(), shared.to(torch.int32).flatten())
    latest = torch.full((count,), -1, dtype=torch.int64, device=DEVICE)
    latest.scatter_reduce_(0, index.flatten(), torch.where(shared, order, -1).flatten(), "amax")
    leaves = shared & ~((writers[index] >= refs[index]) & (latest[index] == order))
    need = inside & (~held | leaves)
    rank = need.flatten().cumsum(0).view(b, columns) - 1
    free = refs == 0
    pages = torch.full((count + 1,), -1, dtype=torch.int32, device=DEVICE)
    pages.scatter_(0, torch.where(free, free.cumsum(0) - 1, count), torch.arange(count, device=DEVICE, dtype=torch.int32))
    short = (need.sum() - free.sum()).clamp(min=0)
    need, leaves = need & (short == 0), leaves & (short == 0)
    fresh = torch.where(need, pages[rank.clamp(min=0, max=count - 1)], -1)
    change(torch.where(leaves, table, -1), -1)
    change(fresh, 1)
    rows = s["lens"] % page
    start = first.long().clamp(max=columns - 1)
    copied = leaves.gather(1, start) & (rows > 0)[:, None]
    copies = torch.where(copied, torch.cat((table.gather(1, start), fresh.gather(1, start), rows[:, None]), 1), -1)
    table.copy_(torch.where(need, fresh, table))

    # What lies behind the tokens that were kept.
    behind = (at >= (s["kept"][:, None] + page - 1) // page) & (table >= 0)
    change(torch.where(behind, table, -1), -1)
    table.masked_fill_(behind, -1)
    return {"table": table, "refs": refs, "copies": copies, "short": short.to(torch.int32).view(1)}


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"probs": _plain_probs, "verify": _plain_verify, "compact": _plain_compact, "copy": _plain_copy,
                "pages": _plain_pages}[op](s)
    af1 = _af1()
    if op == "probs":
        return {"probs": af1.token_probs(s["logits"], temperature=s["temperature"], top_k=s["top_k"], min_p=s["min_p"],
                                         out=s["out"])}
    if op == "verify":
        path, lengths, following = af1.verify_tree(s["probs"], s["tokens"], s["parents"], s["uniforms"], draft=s["draft"],
                                                   counts=s["counts"], distinct=s["case"]["draft"] == "distinct")
        return {"path": path, "lengths": lengths, "following": following}
    if op == "compact":
        af1.kv_compact(s["caches"], s["table"], s["first"], s["index"], s["counts"])
        return _pools(s)
    if op == "copy":
        af1.kv_copy(s["caches"], s["copies"])
        return _pools(s)
    s["pages"].fork(s["parents"])
    copies, short = s["pages"].reserve(s["lens"], s["counts"])
    s["pages"].release(s["kept"])
    return {"table": s["table"], "refs": s["refs"], "copies": copies, "short": short}


# -- the definitions in 64 bits ---------------------------------------------------------


def _exact_row(x, t, k, p):
    """One row: softmax of what the cuts leave."""
    x = x.double()
    y = torch.zeros_like(x)
    if t < 1e-30:
        y[(x == x.max()).nonzero()[0]] = 1.0
        return y
    kept = torch.sort(x, descending=True, stable=True).indices[: k if k > 0 else None]
    share = torch.softmax(x[kept] / t, 0)
    share = torch.where(x[kept] >= x.max() + (t * math.log(p) if p > 0 else -math.inf), share, 0.0)
    y[kept] = share / share.sum()
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "probs":
        t, k, p = (_column(s[x], case["rows"], torch.float32)[:, 0].double().tolist()
                   for x in ("temperature", "top_k", "min_p"))
        return {"probs": torch.stack([_exact_row(s["logits"][i], t[i], int(k[i]), p[i]) for i in range(case["rows"])])}
    if case["op"] in ("compact", "copy"):
        if case["op"] == "copy":
            source, target, rows = s["copies"].T.tolist()
            moves = [(a, i, b, i) for a, b, r in zip(source, target, rows) for i in range(r)]
        else:
            moves, page, table = [], case["page"], s["table"].tolist()
            for b, (first, row, n) in enumerate(zip(s["first"].tolist(), s["index"].tolist(), s["counts"].tolist())):
                for j in range(n):
                    a, z = first + row[j], first + j
                    moves.append((table[b][a // page], a % page, table[b][z // page], z % page))
        moves = torch.tensor(moves, device=DEVICE).view(-1, 4).T
        found = []
        for layer in s["layers"]:
            found.append([])
            for x in layer.values():
                if x is not None:
                    whole = "int" in str(x.dtype)
                    y = x.float().double() if not whole else None
                    if not whole:
                        old = y.clone()
                        y[moves[2], :, moves[3]] = old[moves[0], :, moves[1]]
                    found[-1].append(y)
        return found
    return None  # whole numbers, which comparisons decide
