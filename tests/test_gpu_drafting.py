"""What follows the logits of drafted tokens, against plain restatements in 64
bits and whole numbers: probabilities, verification, accepted slots, copied
pages, the table of pages, and a run of them together."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
I32, F32, F16 = torch.int32, torch.float32, torch.float16
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def P():
    import paper_2609_06161_gb300 as P
    return P


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# -- probabilities -------------------------------------------------------------------


def probs_oracle(x, temperature, top_k, min_p):
    """One row, float64 numpy."""
    x = x.astype(np.float64)
    n = x.size
    if np.isnan(x).any() or (x == INF).any():
        return np.full(n, NAN)
    top = x.max()
    if top == -INF:
        return np.zeros(n)
    y = np.zeros(n)
    if not temperature >= 1e-30:
        y[int(np.argmax(x))] = 1.0
        return y
    temperature = min(temperature, 1e30)
    keep = np.ones(n, bool)
    if 1 <= top_k < n:
        keep[:] = False
        keep[np.argsort(-x, kind="stable")[:top_k]] = True
    share = 0.0 if math.isnan(min_p) else min(max(min_p, 0.0), 1.0)
    if share > 0:
        keep &= x >= top + temperature * math.log(share)
    y[keep] = np.exp((x[keep] - top) / temperature)
    return y / y.sum()


def check_probs(got, x, temperature, top_k, min_p):
    rows, n = x.shape
    col = lambda v: v.double().cpu().numpy() if torch.is_tensor(v) else np.full(rows, float(np.float32(v)))  # noqa: E731
    t, k, m = col(temperature), col(top_k), col(min_p)
    got, x = got.double().cpu().numpy(), x.float().cpu().numpy()
    for r in range(rows):
        want = probs_oracle(x[r], t[r], int(k[r]), m[r])
        assert np.array_equal(np.isnan(got[r]), np.isnan(want)), r
        if np.isnan(want).any():
            continue
        assert (got[r][want == 0] == 0).all() and (got[r][want > 1e-37] > 0).all(), r
        # The exponent d = (x - M) log2(e) / T: three roundings of half a unit, 3 * 2^-24 d ln 2 of the weight; 2^-22 for
        # the power of two; the same of the sum, which adds up to n / 512 + 40 weights one after another, 2^-24 each; 1 / S and
        # the product 2^-24 each. Weights of d above 30 are below 2^-30 of the sum and tell nothing of its error.
        with np.errstate(invalid="ignore"):
            d = np.where(want > 0, np.abs(x[r].astype(np.float64) - np.nanmax(x[r])) / (t[r] if t[r] >= 1e-30 else 1.0) * 1.4427, 0.0)
        tol = 3 * 2.0 ** -24 * 0.6932 * (np.minimum(d, 200) + 30) + 2 * 2.0 ** -22 + (n / 512 + 44) * 2.0 ** -24
        assert (np.abs(got[r] - want) <= tol * want + 2.0 ** -126).all(), (r, np.max(np.abs(got[r] - want) / np.maximum(want, 1e-30)))


def draw_logits(g, rows, vocab, dtype, spread=3.0):
    return (spread * torch.randn((rows, vocab), generator=g, device="cuda")).to(dtype)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 7), (5, 33), (40, 1000), (3, 4097), (700, 515), (2, 32000),
                                        (1, 128001), (2, 300001), (1, 1000003)])
def test_probs_sizes(P, dtype, rows, vocab):
    g = gen(vocab)
    x = draw_logits(g, rows, vocab, dtype)
    for kw in (dict(), dict(temperature=0.7, top_k=max(1, vocab // 3), min_p=0.01), dict(temperature=1.3, min_p=0.2),
               dict(top_k=1), dict(temperature=0.0)):
        full = dict(temperature=1.0, top_k=0, min_p=0.0) | kw
        check_probs(P.token_probs(x, **kw), x, **full)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("vocab", [6, 1003, 40000])
def test_probs_rows_of_their_own(P, dtype, vocab):
    """Each row has its settings, those that say nothing or lie outside their range among them."""
    g = gen(vocab + 1)
    rows = 24
    x = draw_logits(g, rows, vocab, dtype)
    t = torch.tensor([0.0, 1.0, 0.5, 2.0, 1e-30, 1e30, 1e-38, INF, NAN, -1.0, 0.9, 0.3] * 2, device="cuda")
    k = torch.tensor([0, 1, 2, 5, vocab - 1, vocab, vocab + 1, -3, 2 ** 31 - 1, -2 ** 31, vocab // 2, 3] * 2, dtype=I32,
                     device="cuda").roll(5)
    m = torch.tensor([0.0, 0.5, 1.0, 2.0, -1.0, NAN, 1e-30, 0.05] * 3, device="cuda")
    check_probs(P.token_probs(x, t, k, m), x, t, k, m)
    again = P.token_probs(x, t, k, m)
    assert torch.equal(again.nan_to_num(7), P.token_probs(x, t, k, m).nan_to_num(7))  # to the bit


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("vocab,levels", [(50, 1), (50, 4), (5000, 1), (5000, 3), (128001, 1), (128001, 7)])
def test_probs_ties(P, dtype, vocab, levels):
    """Equal entries go by index, across the stretches of a row."""
    g = gen(levels)
    x = torch.randint(0, levels, (8, vocab), generator=g, device="cuda").to(dtype) - 2
    x[:, ::3] *= -0.0 if levels == 1 else 1.0
    k = torch.tensor([1, 2, vocab // 7 + 1, vocab // 2, vocab - 1, vocab, 3, 17], dtype=I32, device="cuda")
    m = torch.tensor([0.0, 1.0, 0.0, 0.1, 0.0, 0.5, 0.0, 1.0], device="cuda")
    check_probs(P.token_probs(x, 1.0, k, m), x, 1.0, k, m)
    check_probs(P.token_probs(x, 0.0, k, m), x, 0.0, k, m)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("vocab", [9, 2500, 70001])
def test_probs_infinities(P, dtype, vocab):
    g = gen(3)
    x = draw_logits(g, 12, vocab, dtype)
    x[0] = -INF
    x[1] = -INF
    x[1, vocab // 2] = -3.0
    x[2, vocab - 1] = NAN
    x[3, 0] = INF
    x[4, ::2] = -INF
    x[5] = torch.finfo(dtype).min
    x[6] = torch.finfo(dtype).min
    x[6, 3] = torch.finfo(dtype).max
    x[7, :] = -INF
    x[7, :3] = 1.0
    x[8, :] = -INF
    x[8, 4] = NAN
    for kw in (dict(temperature=1.0, top_k=0, min_p=0.0), dict(temperature=0.1, top_k=5, min_p=0.0),
               dict(temperature=2.0, top_k=vocab - 1, min_p=0.01), dict(temperature=0.0, top_k=2, min_p=0.5)):
        check_probs(P.token_probs(x, **kw), x, **kw)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("shift,out_shift", [(0, 0), (1, 1), (3, 3), (1, 2), (5, 1), (7, 3)])
def test_probs_strides(P, dtype, shift, out_shift):
    """Rows at any element of a larger tensor; what lies between them stays."""
    g = gen(shift)
    vocab = 2011
    big = draw_logits(g, 6, vocab + 13, dtype)
    x = big[:, shift: shift + vocab]
    out = torch.full((6, vocab + 9), -7.0, device="cuda")
    y = out[:, out_shift: out_shift + vocab]
    kw = dict(temperature=0.8, top_k=100, min_p=0.001)
    assert P.token_probs(x, out=y, **kw) is y
    check_probs(y, x, **kw)
    assert (out[:, :out_shift] == -7).all() and (out[:, out_shift + vocab:] == -7).all()


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("vocab", [16500, 34000, 50001, 128001])
@pytest.mark.parametrize("order", ["any", "rising", "falling"])
def test_probs_many_rows(P, dtype, vocab, order):
    """Calls of more rows than the GPU takes at once in parts, each with its settings; largest entries early and late; ties,
    infinities and rows of few entries among them."""
    g = gen(vocab)
    rows = 320
    x = draw_logits(g, rows, vocab, F32)
    if order != "any":
        x[::2] = x[::2].sort(dim=-1, descending=order == "falling").values
    x[3::16] = (x[3::16] * 2).round() / 2
    x[5::16] = torch.where(torch.rand(x[5::16].shape, generator=g, device="cuda") < 0.997, -INF, x[5::16])
    x[6, vocab // 2], x[7, 3], x[8], x[9, 1:] = NAN, INF, -INF, -INF
    x[10] = 1.0
    x = x.to(dtype)
    t = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, 0.0, 0.5 + torch.rand(rows, generator=g, device="cuda"))
    k = torch.tensor([0, 1, 7, 50, 200, 255, 256, 257, 400, 700, 1000, 1023, 1024, 1500, vocab // 2, vocab - 1], dtype=I32,
                     device="cuda")[torch.randint(0, 16, (rows,), generator=g, device="cuda")]
    m = torch.tensor([0.0, 0.0, 0.5, 0.05, 1e-3, 1e-8], device="cuda")[torch.randint(0, 6, (rows,), generator=g, device="cuda")]
    out = torch.full((rows, vocab + 3), -7.0, device="cuda")
    y = P.token_probs(x, t, k, m, out=out[:, 1: vocab + 1])
    check_probs(y, x, t, k, m)
    assert (out[:, 0] == -7).all() and (out[:, vocab + 1:] == -7).all()
    again = P.token_probs(x, t, k, m)
    assert torch.equal(again.nan_to_num(7), y.nan_to_num(7))


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("vocab", [700, 3000, 20011, 128001, 700001])
def test_probs_large_k(P, dtype, vocab):
    """More entries than the lists hold: among spread values, values that crowd in one place of a wide range, many equal
    ones, and rows with few entries that are not banned."""
    g = gen(vocab)
    x = draw_logits(g, 6, vocab, F32)
    x[1] = torch.where(x[1] > 2, 1e4 * x[1], 1e-3 * x[1])
    x[2] = (x[2] * 2).round() / 2
    x[3, torch.rand(vocab, generator=g, device="cuda") < 0.9] = -INF
    x[4] = 0.25
    x[4, 5], x[4, vocab - 2] = 30.0, -1e4
    x[5] = torch.where(x[5] > 0, 3e38, -3e38) if dtype == F32 else torch.where(x[5] > 0, 6e4, -6e4)
    x = x.to(dtype)
    for k in (257, vocab // 3, vocab // 2, vocab - 1):
        for m in (0.0, 1e-3):
            check_probs(P.token_probs(x, 1.1, k, m), x, 1.1, k, m)


@pytest.mark.parametrize("rows,vocab", [(3, 5), (24, 1003), (320, 40000), (48, 128001), (6, 500003)])
@pytest.mark.parametrize("shift", [0, 1])
def test_probs_in_place(P, rows, vocab, shift):
    """out may be logits: the same results as beside them, whatever is cut; what lies between rows stays."""
    g = gen(vocab)
    big = torch.full((rows, vocab + 3), -7.0, device="cuda")
    x = big[:, shift: shift + vocab]
    start = draw_logits(g, rows, vocab, F32)
    start[-1, vocab // 2:] = -INF
    start[-2, 1] = NAN
    pick = lambda *v: torch.tensor(v, device="cuda")[torch.randint(0, len(v), (rows,), generator=g, device="cuda")]  # noqa: E731
    own = dict(temperature=pick(0.0, 0.7, 1.0, 1.5), top_k=pick(0, 1, 50, 900, vocab // 2).to(I32), min_p=pick(0.0, 0.0, 1e-3, 0.1))
    beside = big.clone()[:, shift: shift + vocab]  # lies as x does, so that its sums are added up in the same order
    for kw in (own, dict(temperature=1.0, top_k=0, min_p=0.0), dict(temperature=0.8, top_k=50, min_p=0.0),
               dict(temperature=0.0, top_k=0, min_p=0.0)):
        x.copy_(start), beside.copy_(start)
        assert P.token_probs(x, out=x, **kw) is x
        check_probs(x, start, **kw)
        assert torch.equal(x.nan_to_num(7), P.token_probs(beside, **kw).nan_to_num(7))
        assert (big[:, :shift] == -7).all() and (big[:, shift + vocab:] == -7).all()


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("k", [0, 40000000])
def test_probs_sums_of_long_rows(P, dtype, k):
    """16000 nearly equal weights for every thread, whose roundings in one long sum would all go one way: that sum would be
    off by 2^-14 or more."""
    vocab, low = (1 << 26) + 3, -0.30859375
    x = torch.full((1, vocab), low, device="cuda").to(dtype)
    x[0, ::1 << 20] = 0.0  # in every stretch of the row
    got = P.token_probs(x, top_k=k)[0]
    kept, tops, rest = k or vocab, 65, math.exp(low)
    top = 1.0 / (tops + (kept - tops) * rest)
    # Three roundings of the exponent d = 0.45 and 2^-22 for its power, of the weight and of the sum's weights; up to 256
    # weights one after another, 2^-24 each, and 60 more for the sums of these, 1 / S and the product.
    tol = 2 * (3 * 2.0 ** -24 * 0.6932 * 0.45 + 2.0 ** -22) + (256 + 60) * 2.0 ** -24
    assert int((got > 0).sum()) == kept
    assert abs(float(got[0]) / top - 1) <= tol
    assert abs(float(got[1]) / (top * rest) - 1) <= tol


def test_probs_cut_next_to_an_entry(P):
    """The bound of min_p in 64 bits: entries a unit in the last place above and below it."""
    t, m = 0.75, 0.05
    bound = 4.0 + t * math.log(float(np.float32(m)))
    least = np.float32(bound) if float(np.float32(bound)) >= bound else np.nextafter(np.float32(bound), np.float32(9))
    x = torch.full((1, 300), -20.0, device="cuda")
    x[0, 7], x[0, 100] = 4.0, float(least)
    x[0, 200] = float(np.nextafter(least, np.float32(-9)))
    p = P.token_probs(x, t, 0, m)[0]
    assert p[7] > 0 and p[100] > 0 and p[200] == 0 and int((p > 0).sum()) == 2


# -- verification --------------------------------------------------------------------


UNIT = 2.0 ** 40


def verify_oracle(probs, tokens, parents, u, draft, count, distinct):
    """One sequence, as the header defines it: numpy, float32 and float64."""
    f32, f64 = np.float32, np.float64
    vocab = probs.shape[1]
    if count <= 0:
        return [], -1
    clean = lambda r: np.clip(np.where(np.isnan(r), f32(0), r), f32(0), f32(1)).astype(f32)  # noqa: E731
    at, path = 0, [0]

    def masses(c, gone):
        r = clean(probs[at])
        if draft is not None:
            r = np.maximum(r - (f32(c) * clean(draft[at])).astype(f32), f32(0)).astype(f32)
        m = np.rint(r.astype(f64) * UNIT).astype(np.int64)
        m[sorted(gone)] = 0
        return m

    while True:
        c, z, zq, gone, taken = f64(0), f64(1), f64(1), set(), None
        for i in range(1, count):
            x = int(tokens[i])
            if parents[i] != at or not 0 <= x < vocab:
                continue
            p = clean(probs[at, x])
            if draft is None:
                r = f64(0) if x in gone else f64(p)
                if f64(u[i]) * z < r:
                    taken = i
                    break
                z = z - r
                gone.add(x)
                continue
            if not zq > 0 or (distinct and x in gone):
                continue
            q = clean(draft[at, x])
            r = f64(0) if x in gone else f64(np.maximum(p - f32(f32(c) * q), f32(0)))
            if f64(u[i]) * f64(q) * z < r * zq:
                taken = i
                break
            c = c + z / zq
            if distinct:
                zq = zq - f64(q)
            gone.add(x)
            z = f64(int(masses(c, gone).sum())) / UNIT
        if taken is None:
            break
        at = taken
        path.append(at)
    m = masses(c if draft is not None else 0.0, gone)
    if m.sum() == 0:
        c, draft = f64(0), None
        m = masses(c, set())
    if m.sum() == 0:
        return path, -1
    w = f64(0) if np.isnan(u[0]) else min(max(f64(u[0]), 0.0), 1 - 2.0 ** -24)
    bound = int(math.floor(w * f64(int(m.sum()))))
    return path, int(np.searchsorted(np.cumsum(m), bound, side="right"))


def check_verify(P, probs, tokens, parents, u, draft=None, counts=None, distinct=False):
    path, lengths, following = P.verify_tree(probs, tokens, parents, u, draft=draft, counts=counts, distinct=distinct)
    b, n = tokens.shape
    c = lambda x: None if x is None else x.cpu().numpy()  # noqa: E731
    args = [c(x) for x in (probs, tokens, parents, u, draft)]
    for s in range(b):
        count = n if counts is None else min(n, int(counts[s]))
        want, token = verify_oracle(*[None if x is None else x[s] for x in args], count, distinct)
        got = path[s].tolist()
        assert got == want + [-1] * (n - len(want)), (s, got, want)
        assert int(lengths[s]) == len(want), s
        assert int(following[s]) == token, (s, int(following[s]), token)
    return path, lengths, following


def trees(rng, b, n, chain=False):
    return torch.tensor([[-1 if i == 0 else i - 1 if chain else int(rng.integers(0, i)) for i in range(n)] for _ in range(b)],
                        dtype=I32, device="cuda")


def distributions(g, b, n, vocab, near, spread=2.0):
    x = spread * torch.randn((b, n, vocab), generator=g, device="cuda")
    y = x + near * torch.randn((b, n, vocab), generator=g, device="cuda")
    return torch.softmax(x, -1), torch.softmax(y, -1)


def drawn_tokens(g, draft, parents, distinct):
    """Children drawn from their parents' rows, in order."""
    b, n, vocab = draft.shape
    per = min(n, vocab)
    drawn = torch.multinomial(draft.view(b * n, vocab), per, replacement=not distinct, generator=g).view(b, n, per)
    up = parents.clamp(min=0).tolist()
    place = torch.tensor([[row[:i].count(row[i]) - (row[i] == 0) for i in range(n)] for row in up], device="cuda").clamp(0, per - 1)
    seq = torch.arange(b, device="cuda")[:, None]
    return drawn[seq, parents.long().clamp(min=0), place].to(I32)


@pytest.mark.parametrize("mode", ["drawn", "distinct", "guessed"])
@pytest.mark.parametrize("b,n,vocab", [(1, 1, 1), (3, 2, 1), (2, 5, 2), (4, 8, 5), (6, 64, 37), (5, 6, 1000), (3, 7, 4096),
                                       (2, 12, 32001), (40, 4, 515), (1, 6, 128001), (400, 3, 130), (20, 3, 70001),
                                       (320, 2, 3001), (1, 3, 1 << 22), (9, 2, 300007)])
def test_verify_sizes(P, mode, b, n, vocab):
    g, rng = gen(b * 1000 + n), np.random.default_rng(n)
    probs, draft = distributions(g, b, n, vocab, 0.7)
    parents = trees(rng, b, n, chain=n == 6)
    tokens = drawn_tokens(g, draft, parents, mode == "distinct")
    u = torch.rand((b, n), generator=g, device="cuda")
    check_verify(P, probs, tokens, parents, u, None if mode == "guessed" else draft, distinct=mode == "distinct")
    counts = torch.randint(-1, n + 2, (b,), generator=g, device="cuda", dtype=I32)
    check_verify(P, probs, tokens, parents, u, None if mode == "guessed" else draft, counts, mode == "distinct")


@pytest.mark.parametrize("mode", ["drawn", "distinct", "guessed"])
def test_verify_wide_trees(P, mode):
    """All nodes are children of the root: many rejections at one node, one accepted late, then its children."""
    g = gen(5)
    b, n, vocab = 64, 40, 64
    probs, draft = distributions(g, b, n, vocab, 3.0)
    parents = torch.zeros((b, n), dtype=I32, device="cuda")
    parents[:, 0] = -1
    parents[:, 30:] = torch.randint(1, 30, (b, 10), generator=g, device="cuda", dtype=I32)
    tokens = drawn_tokens(g, draft, parents, mode == "distinct")
    u = torch.rand((b, n), generator=g, device="cuda")
    u[::2] = 0.5 + 0.5 * u[::2]
    _, lengths, _ = check_verify(P, probs, tokens, parents, u, None if mode == "guessed" else draft,
                                 distinct=mode == "distinct")
    assert (lengths > 1).any()


@pytest.mark.parametrize("mode", ["drawn", "distinct", "guessed"])
def test_verify_odd_trees(P, mode):
    """Parents behind their children, no node's, their own or in a ring; tokens outside the vocabulary or twice; numbers
    that are none."""
    g, rng = gen(6), np.random.default_rng(6)
    b, n, vocab = 96, 10, 12
    probs, draft = distributions(g, b, n, vocab, 1.0)
    parents = torch.tensor(rng.integers(-2, n + 2, (b, n)), dtype=I32, device="cuda")
    parents[:, ::3] = 0
    parents[::5, 1], parents[::5, 2] = 2, 1
    tokens = torch.tensor(rng.integers(-2, vocab + 2, (b, n)), dtype=I32, device="cuda")
    u = torch.rand((b, n), generator=g, device="cuda")
    u[3::7, 0], u[4::7, 1:] = NAN, NAN
    u[5::7, 0], u[6::7, 0] = 1.0, -1.0
    u[::4, 0] = 0.0
    u[1::4, 0] = 1 - 2.0 ** -24
    check_verify(P, probs, tokens, parents, u, None if mode == "guessed" else draft, distinct=mode == "distinct")


@pytest.mark.parametrize("mode", ["drawn", "distinct", "guessed"])
def test_verify_odd_rows(P, mode):
    """Rows without mass, with NaN, infinities and entries outside 0 .. 1; a draft that is the target; certain tokens."""
    g, rng = gen(7), np.random.default_rng(7)
    b, n, vocab = 60, 6, 700
    probs, draft = distributions(g, b, n, vocab, 1.0)
    parents = trees(rng, b, n)
    tokens = drawn_tokens(g, draft, parents, mode == "distinct")
    probs[0:5] = 0.0
    draft[5:10] = probs[5:10]
    probs[10:15] = torch.nn.functional.one_hot(torch.randint(0, vocab, (5, n), generator=g, device="cuda"), vocab).float()
    draft[15:20] = torch.nn.functional.one_hot(torch.randint(0, vocab, (5, n), generator=g, device="cuda"), vocab).float()
    probs[20:25, :, ::3] = NAN
    draft[25:30, :, ::3] = NAN
    probs[30:33, :, 5], probs[33:35, :, 5] = INF, -INF
    draft[35:38, :, 9], draft[38:40, :, 9] = INF, -INF
    probs[40:45] = 1.0
    draft[45:50] = 0.0
    draft[50:55] = 1.0
    probs[55:60] = 2.0 ** -42  # below half a unit of mass
    u = torch.rand((b, n), generator=g, device="cuda")
    check_verify(P, probs, tokens, parents, u, None if mode == "guessed" else draft, distinct=mode == "distinct")


@pytest.mark.parametrize("pad,draft_pad,shift,draft_shift", [(0, 0, 1, 1), (3, 3, 0, 0), (1, 2, 2, 3), (0, 5, 3, 0)])
def test_verify_strides(P, pad, draft_pad, shift, draft_shift):
    g, rng = gen(8), np.random.default_rng(8)
    b, n, vocab = 5, 9, 1501
    p, q = distributions(g, b, n, vocab, 0.7)
    at = lambda x, pad, shift: torch.cat((torch.full((b, n, shift), NAN, device="cuda"), x, torch.full(  # noqa: E731
        (b, n, pad), NAN, device="cuda")), -1)[..., shift: shift + vocab]
    parents = trees(rng, b, n)
    tokens = drawn_tokens(g, q, parents, False)
    u = torch.rand((b, n), generator=g, device="cuda")
    check_verify(P, at(p, pad, shift), tokens, parents, u, at(q, draft_pad, draft_shift))
    turned = p.transpose(0, 1).contiguous().transpose(0, 1)
    check_verify(P, turned, tokens, parents, u, q[:1].expand(b, -1, -1))  # one draft for all sequences


@pytest.mark.parametrize("mode", ["drawn", "distinct", "guessed"])
def test_verify_rows_off_the_path(P, mode):
    """What lies in rows of nodes that the walk does not come to changes nothing."""
    g, rng = gen(16), np.random.default_rng(16)
    b, n, vocab = 12, 14, 700
    probs, draft = distributions(g, b, n, vocab, 0.7)
    parents = trees(rng, b, n)
    tokens = drawn_tokens(g, draft, parents, mode == "distinct")
    u = torch.rand((b, n), generator=g, device="cuda")
    kw = dict(draft=None if mode == "guessed" else draft, distinct=mode == "distinct")
    want = P.verify_tree(probs, tokens, parents, u, **kw)
    on = torch.zeros((b, n + 1), dtype=torch.bool, device="cuda").scatter_(1, torch.where(want[0] < 0, n, want[0]).long(), True)
    for t, other in ((probs, NAN), (draft, INF), (probs, 1.0), (draft, -INF)):
        t[~on[:, :n]] = other
        assert all(torch.equal(a, z) for a, z in zip(P.verify_tree(probs, tokens, parents, u, **kw), want))


@pytest.mark.parametrize("mode", ["drawn", "distinct", "guessed"])
def test_verified_tokens_have_the_targets_distribution(P, mode):
    """Many sequences with one target and one draft: the first token that comes out (an accepted child's or the one that
    follows) has the target's probabilities, within 6 standard deviations."""
    g = gen(9)
    b, n, vocab = 60000, 5, 11
    p, q = (torch.softmax(torch.randn(vocab, generator=g, device="cuda") * s, 0) for s in (1.0, 1.3))
    parents = torch.tensor([-1, 0, 0, 0, 0], dtype=I32, device="cuda").repeat(b, 1)
    if mode == "guessed":
        tokens = torch.tensor([0, 3, 7, 3, 1], dtype=I32, device="cuda").repeat(b, 1)
    else:
        drawn = torch.multinomial(q.expand(b, -1), n - 1, replacement=mode == "drawn", generator=g).to(I32)
        tokens = torch.cat((torch.zeros((b, 1), dtype=I32, device="cuda"), drawn), 1)
    u = torch.rand((b, n), generator=g, device="cuda")
    shape = lambda x: x.expand(b, n, vocab)  # noqa: E731
    path, lengths, following = P.verify_tree(shape(p), tokens, parents, u, draft=None if mode == "guessed" else shape(q),
                                             distinct=mode == "distinct")
    first = torch.where(lengths > 1, tokens.gather(1, path[:, 1:2].long().clamp(min=0))[:, 0], following)
    share = torch.bincount(first.long(), minlength=vocab).double() / b
    p = p.double()
    assert ((share - p).abs() <= 6 * (p * (1 - p) / b).sqrt()).all(), (share, p)
    accepted = float((lengths > 1).double().mean())
    if mode == "guessed":  # the share of the guesses themselves
        want = float(p[[1, 3, 7]].sum())
        assert abs(accepted - want) <= 6 * math.sqrt(want * (1 - want) / b)
    else:  # at least the overlap of the two distributions
        want = float(torch.minimum(p, q.double()).sum())
        assert accepted >= want - 6 * math.sqrt(want * (1 - want) / b)


def test_verify_greedy(P):
    """One-hot rows: the path is what greedy decoding takes."""
    g = gen(10)
    b, n, vocab = 20, 12, 300
    logits = torch.randn((b, n, vocab), generator=g, device="cuda")
    probs = P.token_probs(logits.view(b * n, vocab), temperature=0.0).view(b, n, vocab)
    best = logits.argmax(-1)
    parents = trees(np.random.default_rng(1), b, n)
    tokens = best.gather(1, parents.long().clamp(min=0)).to(I32)
    tokens[:, ::2] = torch.randint(0, vocab, (b, n // 2), generator=g, device="cuda", dtype=I32)
    u = torch.rand((b, n), generator=g, device="cuda")
    path, lengths, following = check_verify(P, probs, tokens, parents, u)
    given = tuple(torch.full_like(t, 7) for t in (path, lengths, following))
    assert all(a is z for a, z in zip(P.verify_tree(probs, tokens, parents, u, out=given), given))
    assert all(torch.equal(a, z) for a, z in zip(given, (path, lengths, following)))
    last = path.gather(1, (lengths[:, None] - 1).long())
    assert torch.equal(following, best.gather(1, last.long())[:, 0].to(I32))


# -- accepted slots and copied pages -------------------------------------------------


KINDS = ["f16", "int8", "e4m3", "int4"]


def bits(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16 if x.element_size() == 2 else I32)


def filled(P, g, kind, pages, page, heads, dim):
    c = P.KVCache.empty(pages, page, heads, dim, kind)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        if t is not None:
            b = bits(t)
            b.copy_(torch.randint(0, 100, b.shape, generator=g, device="cuda", dtype=b.dtype))
    return c


def parts(c):
    return [bits(t) for t in (c.k, c.v, c.k_scale, c.v_scale) if t is not None]


def compact_oracle(c, pages, first, index, counts):
    out = [t.cpu().numpy().copy() for t in parts(c)]
    old = [t.copy() for t in out]
    pages, index = pages.cpu().numpy(), index.cpu().numpy()
    rows, columns = pages.shape

    def row(s, slot):
        if slot < 0 or slot // c.page_size >= columns:
            return None
        page = pages[s, slot // c.page_size]
        return (page, slot % c.page_size) if 0 <= page < c.pages else None

    for s in range(rows):
        for j in range(min(index.shape[1], int(counts[s]))):
            a, z = row(s, int(first[s]) + int(index[s, j])), row(s, int(first[s]) + j)
            if a is None or z is None:
                continue
            for new, was in zip(out, old):
                new[z[0], :, z[1]] = was[a[0], :, a[1]]
    return out


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,page,heads,nodes", [(64, 16, 1, 1), (64, 32, 3, 9), (128, 16, 2, 64), (128, 128, 8, 17),
                                                  (64, 256, 5, 33)])
@pytest.mark.parametrize("order", ["path", "any"])
def test_compact(P, kind, dim, page, heads, nodes, order):
    g, rng = gen(nodes), np.random.default_rng(nodes)
    b = 7
    columns = (100 + nodes) // page + 2
    caches = [filled(P, g, kind, b * columns + 3, page, heads, dim), filled(P, g, "f16", b * columns, page, 1, 128)]
    pages = torch.tensor(rng.permutation(b * columns).reshape(b, columns), dtype=I32, device="cuda")
    first = torch.tensor([0, 1, 99, page - 1, page, 50, 3], dtype=I32, device="cuda")
    if order == "path":
        index = [[0] + sorted(rng.choice(nodes - 1, nodes - 1, replace=False) + 1)[: nodes - 1] for _ in range(b)]
        index = [[x + (1 if x > nodes // 3 and x < nodes - 1 else 0) for x in row] for row in index]
    else:  # repeated, backwards, behind the nodes
        index = rng.integers(-2, nodes + 20, (b, nodes))
        index[0] = np.arange(nodes)[::-1]
        index[1] = 0
    index = torch.tensor(np.array(index), dtype=I32, device="cuda")
    counts = torch.tensor([nodes, 0, nodes, nodes // 2, nodes + 5, -3, 1], dtype=I32, device="cuda")
    want = [compact_oracle(c, pages, first, index, counts) for c in caches]
    P.kv_compact(caches, pages, first, index, counts)
    for c, w in zip(caches, want):
        for got, x in zip(parts(c), w):
            assert np.array_equal(got.cpu().numpy(), x)


def test_compact_bad_slots(P):
    """Slots and pages outside the table and the cache, of either end of a move, one cache smaller than the other."""
    g, rng = gen(11), np.random.default_rng(11)
    b, columns, nodes = 9, 4, 12
    caches = [filled(P, g, "int8", 40, 16, 2, 64), filled(P, g, "int4", 20, 16, 3, 128)]
    big = torch.full((b, columns + 3), 5, dtype=I32, device="cuda")
    pages = big[:, 1: 1 + columns]
    pages.copy_(torch.tensor(rng.permutation(36).reshape(b, columns)))
    pages[0, 1], pages[1, 1], pages[2, 0], pages[3] = -1, 40, 2 ** 31 - 1, -2 ** 31
    first = torch.tensor([8, 10, 12, 0, -5, 60, 64, 2 ** 31 - 2, -2 ** 31], dtype=I32, device="cuda")
    index = torch.tensor(rng.integers(0, 30, (b, nodes)), dtype=I32, device="cuda")
    index[5, 3], index[6, 2] = 2 ** 31 - 1, -2 ** 31
    counts = torch.full((b,), nodes, dtype=I32, device="cuda")
    want = [compact_oracle(c, pages, first, index, counts) for c in caches]
    P.kv_compact(caches, pages, first, index, counts)
    for c, w in zip(caches, want):
        for got, x in zip(parts(c), w):
            assert np.array_equal(got.cpu().numpy(), x)


@pytest.mark.parametrize("order", ["path", "any"])
@pytest.mark.parametrize("layers,heads", [(12, 7), (40, 7), (40, 8)])
def test_compact_many_layers(P, layers, heads, order):
    """A model's layers, of different heads, in one call."""
    g, rng = gen(layers), np.random.default_rng(layers)
    b, nodes, columns = 60, 21, 5
    caches = [filled(P, g, KINDS[i % 4], b * columns, 16, heads - 4 * (i % 5 == 3), 64) for i in range(layers)]
    pages = torch.tensor(rng.permutation(b * columns).reshape(b, columns), dtype=I32, device="cuda")
    first = torch.tensor(rng.integers(0, 55, b), dtype=I32, device="cuda")
    index = np.sort(rng.permuted(np.tile(np.arange(1, nodes), (b, 1)), axis=1)[:, :9], axis=1)
    index = np.concatenate((np.zeros((b, 1), np.int64), index, np.full((b, nodes - 10), -1)), 1)
    if order == "any":
        index[::2, :10] = index[::2, 9::-1]
    index = torch.tensor(index, dtype=I32, device="cuda")
    counts = torch.tensor(rng.integers(0, 11, b), dtype=I32, device="cuda")
    want = [compact_oracle(c, pages, first, index, counts) for c in caches]
    P.kv_compact(caches, pages, first, index, counts)
    for c, w in zip(caches, want):
        for got, x in zip(parts(c), w):
            assert np.array_equal(got.cpu().numpy(), x)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,page,heads", [(64, 16, 1), (128, 16, 8), (64, 64, 3), (128, 256, 2)])
def test_copy(P, kind, dim, page, heads):
    g = gen(page)
    caches = [filled(P, g, kind, 50, page, heads, dim), filled(P, g, "int8", 60, page, 4, 64)]
    rows = [page, 1, 2, 3, 5, page - 1, page + 7, 0, -4, page // 2, page, page, page, page, 2 ** 31 - 1]
    copies = torch.tensor([[i, 20 + i, r] for i, r in enumerate(rows)], dtype=I32, device="cuda")
    copies[10, 0], copies[11, 1], copies[12, 0], copies[13, 1] = -1, 60, 2 ** 31 - 1, -2 ** 31
    copies[9, 1] = copies[9, 0]
    copies[8, 0] = 55  # in one of the caches alone
    copies[8, 2] = page
    want = []
    for c in caches:
        w = [t.cpu().numpy().copy() for t in parts(c)]
        for a, z, r in copies.tolist():
            if 0 <= a < c.pages and 0 <= z < c.pages and r > 0:
                for t in w:
                    t[z, :, : min(r, page)] = t[a, :, : min(r, page)]
        want.append(w)
    P.kv_copy(caches, copies)
    for c, w in zip(caches, want):
        for got, x in zip(parts(c), w):
            assert np.array_equal(got.cpu().numpy(), x)


def test_many_caches(P):
    """More layers than one launch takes, in two calls at once on one list; refusals that need a cache."""
    g = gen(12)
    caches = [filled(P, g, KINDS[i % 4], 6, 16, 1 + i % 3, 64) for i in range(130)]
    pages = torch.arange(6, dtype=I32, device="cuda").view(1, 6)
    one = lambda *v: torch.tensor(v, dtype=I32, device="cuda")  # noqa: E731
    want = [compact_oracle(c, pages, one(14), one(0, 3, 4).view(1, 3), one(3)) for c in caches]
    for w in want:
        for t in w:
            t[5, :, :9] = t[0, :, :9]
    P.kv_compact(caches, pages, one(14), one(0, 3, 4).view(1, 3), one(3))
    P.kv_copy(caches, one(0, 5, 9).view(1, 3))
    for c, w in zip(caches, want):
        for got, x in zip(parts(c), w):
            assert np.array_equal(got.cpu().numpy(), x)
    other = P.KVCache.empty(6, 32, 1, 64, "f16")
    for bad in ([caches[0], other], [caches[0], caches[1], caches[0]], [],
                [caches[0], P.KVCache(caches[12].k, caches[0].v)]):
        with pytest.raises(P.AF1Error):
            P.kv_copy(bad, one(0, 5, 9).view(1, 3))
        with pytest.raises(P.AF1Error):
            P.kv_compact(bad, pages, one(0), one(0).view(1, 1), one(1))
    gone = P.KVCache.empty(6, 16, 1, 64, "f16")
    gone.free()
    with pytest.raises(P.AF1Error):
        P.kv_copy(gone, one(0, 5, 9).view(1, 3))
    P.kv_copy(caches, torch.zeros((0, 3), dtype=I32, device="cuda"))
    P.kv_compact(caches, pages[:0], one()[:0], torch.zeros((0, 3), dtype=I32, device="cuda"), one()[:0])


# -- the table -----------------------------------------------------------------------


def reserve_oracle(table, refs, page, first, counts):
    """Entry after entry, in order."""
    t, r = table.copy(), refs.copy()
    seqs, columns = t.shape
    holders = lambda e: 0 <= e < r.size  # noqa: E731
    copies, free, lacking = np.full((seqs, 3), -1), [int(x) for x in np.flatnonzero(r == 0)], 0
    for s in range(seqs):
        if first[s] < 0 or counts[s] < 1:
            continue
        for c in range(first[s] // page, min(columns, (int(first[s]) + int(counts[s]) - 1) // page + 1)):
            old = t[s, c]
            if holders(old) and r[old] <= 1:
                continue
            if holders(old):
                r[old] -= 1
            if not free:
                lacking += 1
                continue
            new = free.pop(0)
            t[s, c], r[new] = new, 1
            if holders(old) and c == first[s] // page and first[s] % page:
                copies[s] = old, new, first[s] % page
    if lacking:
        return np.where((table >= 0) & (table < r.size), table, -1), refs, np.full((seqs, 3), -1), lacking
    return t, r, copies, 0


def counted(table, pages):
    inside = table[(table >= 0) & (table < pages)]
    return torch.bincount(inside.long().flatten(), minlength=pages).to(I32)


def random_table(rng, seqs, columns, pages, page, shared=0.5):
    """Rows that share pages in any pattern."""
    t = np.full((seqs, columns), -1, np.int64)
    lens = rng.integers(0, columns * page + 1, seqs)
    pool = rng.permutation(pages)[: max(1, pages // 2)]
    for s in range(seqs):
        n = -(-int(lens[s]) // page)
        t[s, :n] = rng.choice(pool, n)
        if rng.random() < shared and s:
            m = int(rng.integers(0, n + 1))
            o = int(rng.integers(0, s))
            t[s, :m] = np.where(t[o, :m] >= 0, t[o, :m], t[s, :m])
    return t, lens


def norm(t, pages):
    return torch.where((t >= 0) & (t < pages), t, -1)


@pytest.mark.parametrize("seqs,columns,pages,page", [(1, 1, 1, 16), (1, 5, 9, 16), (3, 4, 5, 32), (8, 33, 400, 16),
                                                     (64, 40, 3000, 64), (1024, 9, 20000, 256), (33, 300, 5001, 16),
                                                     (17, 6, 70001, 128)])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_table(P, seqs, columns, pages, page, seed):
    """Steps of fork, reserve and release against rules applied entry after entry; now and then pages are lacking."""
    rng = np.random.default_rng(seed + 100 * seqs)
    start, lens = random_table(rng, seqs, columns, pages, page)
    big = torch.full((seqs, columns + seed), -9, dtype=I32, device="cuda")
    table = big[:, :columns]
    table.copy_(torch.tensor(start))
    refs = counted(table, pages)
    t = P.PageTable(table, refs, page)
    dev = lambda x: torch.tensor(np.asarray(x), dtype=I32, device="cuda")  # noqa: E731
    for step in range(5):
        parents = rng.integers(0, seqs, seqs) if step % 2 else np.arange(seqs)
        parents = np.where(rng.random(seqs) < 0.1, rng.choice([-1, seqs, -2 ** 31, 2 ** 31 - 1], seqs), parents)
        was = table.cpu().numpy()
        t.fork(dev(parents))
        ok = (parents >= 0) & (parents < seqs)
        want = np.where(ok[:, None], was[np.where(ok, parents, 0)], -1)
        lens = np.where(ok, lens[np.where(ok, parents, 0)], 0)
        assert np.array_equal(table.cpu().numpy(), want)
        assert torch.equal(refs, counted(table, pages))

        counts = rng.integers(-1, 3 * page, seqs) if step < 4 else np.full(seqs, 2 ** 31 - 1)
        first = np.where(rng.random(seqs) < 0.05, rng.choice([-1, -2 ** 31, 2 ** 31 - 1], seqs), lens)
        want = reserve_oracle(table.cpu().numpy(), refs.cpu().numpy(), page, first, counts)
        copies, lacking = t.reserve(dev(first), dev(counts))
        assert int(lacking[0]) == want[3]
        assert np.array_equal(table.cpu().numpy(), want[0])
        assert np.array_equal(refs.cpu().numpy(), want[1])
        assert np.array_equal(copies.cpu().numpy(), want[2])
        assert torch.equal(refs, counted(table, pages))

        keep = rng.integers(-3, columns * page + 5, seqs)
        was = norm(table, pages).cpu().numpy()
        t.release(dev(keep))
        kept = np.arange(columns) < -(-np.maximum(keep, 0)[:, None] // page)
        assert np.array_equal(table.cpu().numpy(), np.where(kept, was, -1))
        assert torch.equal(refs, counted(table, pages))
        lens = np.minimum(lens, np.maximum(keep, 0))
    assert (big[:, columns:] == -9).all()


def test_table_last_holder(P):
    """Of a page that several write in one call the last keeps it, unless another entry, or the caller, holds it too."""
    table = torch.tensor([[0, 1], [0, 2], [0, 1], [0, 2], [3, 1]], dtype=I32, device="cuda")
    refs = counted(table, 12)
    refs[2] += 1  # the caller's
    t = P.PageTable(table, refs, 16)
    one = lambda *v: torch.tensor(v, dtype=I32, device="cuda")  # noqa: E731
    copies, lacking = t.reserve(one(17, 20, 21, 31, 16), one(1, 1, 1, 1, 0))
    assert lacking.tolist() == [0]
    assert table.tolist() == [[0, 4], [0, 5], [0, 6], [0, 7], [3, 1]]
    assert copies.tolist() == [[1, 4, 1], [2, 5, 4], [1, 6, 5], [2, 7, 15], [-1, -1, -1]]
    assert refs.tolist() == [4, 1, 1, 1, 1, 1, 1, 1, 0, 0, 0, 0]
    copies, _ = t.reserve(one(3, 0, 15, 1, 0), one(1, 1, 1, 1, 0))
    assert table[:, 0].tolist() == [8, 9, 10, 0, 3]
    assert copies.tolist() == [[0, 8, 3], [-1] * 3, [0, 10, 15], [-1] * 3, [-1] * 3]
    assert refs.tolist() == [1] * 11 + [0]


def test_table_entries_that_hold_no_page(P):
    table = torch.tensor([[7, 2 ** 31 - 1, -5, 3], [100, 3, 3, -1]], dtype=I32, device="cuda")
    refs = counted(table, 8)
    assert refs.tolist() == [0, 0, 0, 3, 0, 0, 0, 1]
    t = P.PageTable(table, refs, 16)
    one = lambda *v: torch.tensor(v, dtype=I32, device="cuda")  # noqa: E731
    _, lacking = t.reserve(one(0, 0), one(1000, 16))
    assert lacking.tolist() == [0] and table.tolist() == [[7, 0, 1, 2], [4, 3, 3, -1]]
    assert torch.equal(refs, counted(table, 8))
    t.release(one(0, 17))
    assert table.tolist() == [[-1] * 4, [4, 3, -1, -1]] and refs.tolist() == [0, 0, 0, 1, 1, 0, 0, 0]


def test_empty_table(P):
    t = P.PageTable.empty(0, 4, 3, 16)
    none = torch.zeros(0, dtype=I32, device="cuda")
    t.fork(none)
    t.release(none)
    copies, lacking = t.reserve(none, none)
    assert copies.shape == (0, 3) and lacking.tolist() == [0]


# -- together ------------------------------------------------------------------------


def test_other_devices_and_streams(P):
    """Host tensors are refused; work goes to the stream that is given."""
    with pytest.raises(P.AF1Error):
        P.token_probs(torch.zeros(2, 5))
    with pytest.raises(P.AF1Error):
        P.PageTable(torch.zeros((1, 1), dtype=I32), torch.zeros(1, dtype=I32), 16).release(torch.zeros(1, dtype=I32))
    g = gen(13)
    x = draw_logits(g, 64, 50000, F32)
    plain = P.token_probs(x, 0.8, 100, 0.01)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        slow = x + 0
        for _ in range(20):
            slow = slow * 1.0
    y = P.token_probs(slow, 0.8, 100, 0.01, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, plain)

    # A chain of calls on two streams at once, each on tensors of its own.
    def chain(stream):
        one = lambda *v: torch.tensor(v, dtype=I32, device="cuda")  # noqa: E731
        cache = filled(P, gen(3), "int8", 12, 16, 2, 64)
        table = P.PageTable.empty(2, 5, 12, 16)
        probs, parents, tokens = y[:6].view(2, 3, -1), one(-1, 0, 0, -1, 0, 1).view(2, 3), one(0, 5, 9, 0, 7, 3).view(2, 3)
        u, first, n = torch.full((2, 3), 0.4, device="cuda"), one(0, 0), one(30, 20)
        back = one(0, 0)
        made = torch.cuda.Event()
        made.record()
        if stream is not None:
            stream.wait_event(made)
        table.reserve(first, n, stream=stream)
        table.fork(back, stream=stream)
        copies, _ = table.reserve(n, n, stream=stream)
        P.kv_copy(cache, copies, stream=stream)
        path, lengths, following = P.verify_tree(probs, tokens, parents, u, stream=stream)
        P.kv_compact(cache, table.table, n, path, lengths, stream=stream)
        table.release(n, stream=stream)
        return [path, lengths, following, table.table, table.refs, copies] + parts(cache)

    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    runs = [chain(s) for s in (side, other, None)]
    torch.cuda.synchronize()
    for a, b, c in zip(*runs):
        assert torch.equal(a, c) and torch.equal(b, c)


def test_a_table_made_while_the_current_stream_is_busy(P):
    """Tables made behind work that the current stream still has to do, and used on another stream, which table and refs
    are ordered with: nothing that the table allocates for itself waits for the current stream."""
    one = lambda *v: torch.tensor(v, dtype=I32, device="cuda")  # noqa: E731
    side = torch.cuda.Stream()
    big = torch.zeros(1 << 28, device="cuda")
    first, n = one(3, 5, 2), one(1, 1, 20)
    for work in (0, 100):  # once for what is done at first use
        tables = [one(0, -1, 0, -1, 1, -1).view(3, 2) for _ in range(2)]
        refs = [counted(t, pages) for t, pages in zip(tables, (6, 2))]
        torch.cuda.synchronize()
        for _ in range(work):
            big.mul_(1.0)
        got = [P.PageTable(t, r, 16).reserve(first, n, stream=side) for t, r in zip(tables, refs)]
        torch.cuda.synchronize()
        (copies, lacking), (no_copies, short) = got
        assert copies.tolist() == [[0, 2, 3], [-1] * 3, [-1] * 3] and lacking.tolist() == [0]
        assert tables[0].tolist() == [[2, -1], [0, -1], [1, 3]]
        assert no_copies.tolist() == [[-1] * 3] * 3 and short.tolist() == [2]
        assert tables[1].tolist() == [[0, -1], [0, -1], [1, -1]]


def test_a_step_in_a_graph(P):
    """Reserve, append, attend, probabilities, verification, compaction, release: captured once, replayed on new inputs,
    with the lengths on the device throughout; against the same calls made one by one."""
    g, rng = gen(14), np.random.default_rng(14)
    b, n, vocab, heads, dim, page, layers = 3, 6, 500, 2, 64, 16, 2
    caches = [filled(P, g, kind, 60, page, heads, dim) for kind in ("int8", "f16")]
    for c in caches:
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            if t is not None:
                t.view(torch.uint8).zero_()
    table = P.PageTable.empty(b, 10, 60, page)
    rope = P.rope_table(200, dim)
    lens = torch.tensor([0, 14, 40], dtype=I32, device="cuda")
    table.reserve(torch.zeros_like(lens), lens)
    parents = trees(rng, b, n)
    depth = torch.zeros((b, n), dtype=I32, device="cuda")
    for s in range(b):
        for i in range(1, n):
            depth[s, i] = depth[s, int(parents[s, i])] + 1
    mask = P.tree_mask(parents)
    counts = torch.full((b,), n, dtype=I32, device="cuda")
    seq = torch.arange(b, dtype=I32, device="cuda").repeat_interleave(n)
    node = torch.arange(n, dtype=I32, device="cuda").repeat(b)
    mix = torch.randn((heads * dim, vocab), generator=g, device="cuda") * 0.3
    ins = dict(x=torch.randn((layers, 3, b * n, heads, dim), generator=g, device="cuda").half(),
               tokens=torch.randint(0, vocab, (b, n), generator=g, device="cuda", dtype=I32),
               u=torch.rand((b, n), generator=g, device="cuda"))
    ws = caches[0].make_workspace(torch.empty((b, n, heads, dim), dtype=F16, device="cuda"))
    state = [lens, table.table, table.refs] + [t for c in caches for t in parts(c)]

    def step():
        copies, lacking = table.reserve(lens, counts)
        P.kv_copy(caches, copies)
        slot = lens.repeat_interleave(n) + node
        h = 0
        for i, c in enumerate(caches):
            k, v, q = ins["x"][i]
            q = c.append(k, v, table.table, seq, slot, rope=rope, positions=(lens[:, None] + depth).view(-1), q=q)
            h = h + c.tree_attention(q.view(b, n, heads, dim), table.table, lens, mask=mask, workspace=ws).float()
        probs = P.token_probs(h.reshape(b * n, heads * dim) @ mix, 0.7, 50, 0.001).view(b, n, vocab)
        # Half of the drafted tokens are the row's likeliest.
        tokens = torch.where(ins["u"] < 0.5, probs.argmax(-1).gather(1, parents.long().clamp(min=0)).to(I32), ins["tokens"])
        path, lengths, following = P.verify_tree(probs, tokens, parents, ins["u"])
        P.kv_compact(caches, table.table, lens, path, lengths)
        lens.add_(lengths)
        table.release(lens)
        return path, lengths, following, lacking

    start = [t.clone() for t in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    torch.cuda.synchronize()
    for t, s in zip(state, start):
        t.copy_(s)
    seen = []
    for k in range(4):
        new = dict(x=torch.randn(ins["x"].shape, generator=g, device="cuda").half(),
                   tokens=torch.randint(0, vocab, (b, n), generator=g, device="cuda", dtype=I32),
                   u=torch.rand((b, n), generator=g, device="cuda"))
        for name, t in new.items():
            ins[name].copy_(t)
        before = [t.clone() for t in state]
        graph.replay()
        got = [t.clone() for t in outs] + [t.clone() for t in state]
        for t, s in zip(state, before):
            t.copy_(s)
        want = list(step()) + [t.clone() for t in state]
        for a, z in zip(got, want):
            assert torch.equal(a, z)
        seen.append(got[1])
        assert int(got[3][0]) == 0
        assert torch.equal(table.refs, counted(table.table, 60))
        held = (table.table >= 0).sum(1)
        assert torch.equal(held, (lens.long() + page - 1) // page)
    assert int(torch.stack(seen).max()) > 1  # drafted tokens were accepted
    P.workspace_status(ws)


def test_compacted_path_attends_like_appended_tokens(P):
    """The cache after a tree's append and the compaction of a path is, to the bit, the cache after the path's tokens were
    appended alone."""
    g = gen(15)
    for kind in KINDS:
        a, z = (P.KVCache.empty(4, 16, 2, 64, kind) for _ in "ab")
        pages = torch.tensor([[2, 0, 3, 1]], dtype=I32, device="cuda")
        rope = P.rope_table(64, 64)
        n, first, path = 12, 13, [0, 2, 5, 9]
        k, v = (torch.randn((n, 2, 64), generator=g, device="cuda").half() for _ in "kv")
        depth = torch.tensor([0, 1, 1, 2, 2, 2, 1, 3, 3, 3, 4, 4], dtype=I32, device="cuda")
        seq = lambda m: torch.zeros(m, dtype=I32, device="cuda")  # noqa: E731
        slots = lambda m: first + torch.arange(m, dtype=I32, device="cuda")  # noqa: E731
        a.append(k, v, pages, seq(n), slots(n), rope=rope, positions=first + depth)
        index = torch.tensor([path + [-1] * 8], dtype=I32, device="cuda")
        one = lambda x: torch.tensor([x], dtype=I32, device="cuda")  # noqa: E731
        P.kv_compact(a, pages, one(first), index, one(4))
        z.append(k[path], v[path], pages, seq(4), slots(4), rope=rope)
        for x, y in zip(a.read(pages, one(first + 4)), z.read(pages, one(first + 4))):
            assert torch.equal(x[:, first:], y[:, first:])


@pytest.mark.parametrize("kind", ["int8", "f16"])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
def test_the_example_samples(kind, temperature):
    """At temperature 0 the verified text is the greedy one, until a near tie parts them (as for the example's greedy
    drafts); at another it runs."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    try:
        import draft_verify
    finally:
        sys.path.pop(0)
    plain, found, passes = draft_verify.sample(kind, steps=30, temperature=temperature, say=lambda _: None)
    assert len(found) == 30 and all(0 <= t < 1000 for t in found)
    if temperature == 0.0:
        same = next((i for i, (a, b) in enumerate(zip(plain, found)) if a != b), len(plain))
        assert same >= 20, (plain, found)
        assert passes < 30  # drafts were accepted


# -- offsets beyond 32 bits ------------------------------------------------------------


def test_far_rows(P):
    """Rows of logits and of probabilities more than 2^31 entries apart."""
    g, rng = gen(20), np.random.default_rng(20)
    far, vocab = (1 << 31) + 8, 3001
    big = torch.empty(far + 4 * vocab, device="cuda")
    x = big.as_strided((2, vocab), (far, 1))
    x.copy_(draw_logits(g, 2, vocab, F32))
    kw = dict(temperature=0.9, top_k=30, min_p=0.001)
    check_probs(P.token_probs(x, **kw), x, **kw)
    want = P.token_probs(x.contiguous(), **kw)
    x.copy_(x.clone())
    y = big.as_strided((2, vocab), (far, 1), vocab)
    assert torch.equal(P.token_probs(x, out=y, **kw), want)

    n = 4
    probs, draft = distributions(g, 2, n, vocab // 4, 0.7)
    parents = trees(rng, 2, n)
    tokens = drawn_tokens(g, draft, parents, False)
    u = torch.rand((2, n), generator=g, device="cuda")
    p = big.as_strided((2, n, vocab // 4), (far, vocab // 4, 1))
    p.copy_(probs)
    check_verify(P, p, tokens, parents, u, draft)


def test_far_pages(P):
    """A cache of more than 2^31 bytes of keys."""
    pages, page, heads = 20000, 64, 8
    c = P.KVCache.empty(pages, page, heads, 128, "f16")
    assert c.k.numel() * 2 > 1 << 31
    near = [pages - 1, pages - 2, 0]
    g = gen(21)
    for t in (c.k, c.v):
        for i in near:
            t[i] = torch.randn(t.shape[1:], generator=g, device="cuda").half()
    one = lambda *v: torch.tensor(v, dtype=I32, device="cuda")  # noqa: E731
    want = [t[near].clone() for t in (c.k, c.v)]
    P.kv_copy(c, one(pages - 1, 0, 40).view(1, 3))
    for w in want:
        w[2, :, :40] = w[0, :, :40]
    P.kv_compact(c, one(pages - 1, pages - 2).view(1, 2), one(60), one(0, 2, 9, 5).view(1, 4), one(4))
    for t, w in zip((c.k, c.v), want):
        was = w.clone()
        w[0, :, 61], w[0, :, 62], w[0, :, 63] = was[0, :, 62], was[1, :, 5], was[1, :, 1]
        assert torch.equal(t[near], w)
        assert float(t[1: pages - 2].abs().max()) == 0
