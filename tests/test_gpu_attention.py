"""Rotary positions, the paged cache, attention of drafted tokens and token
scores against their definitions in 64 bits.

Tolerances come from the arithmetic, u = 2^-11 for FP16 and e = 2^-24 for FP32:
rotations are two products and a sum (3 e of |a| + |b|); stored codes are
compared bit for bit with the same steps in numpy's FP32; for attention, FP16
weights give u sum p|v|, 4-bit entries another u for the values and u sum |q||k|
for the scores, FP32 sums of `dim` products 2 e dim sum |q||k| for the scores,
and the FP16 output u |o|."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

KINDS = ["f16", "int8", "e4m3", "int4"]
U, E = 2.0 ** -11, 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    import paper_2609_06161_gb300 as P
    return P


def gen(seed):
    return np.random.default_rng(seed)


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


# -- definitions -----------------------------------------------------------------


def table_np(length, dim, base=10000.0):
    angle = np.arange(length)[:, None] * base ** (-np.arange(0, dim, 2) / dim)
    return np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)


def pairs(dim, interleaved):
    i = np.arange(dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + dim // 2)


def rotate(x, pos, table, interleaved, dtype, sign=1):
    """x (tokens, heads, dim) in `dtype` arithmetic, each operation rounded."""
    y = x.astype(dtype)
    first, second = pairs(2 * table.shape[1], interleaved)
    c, s = table[pos, None, :, 0].astype(dtype), dtype(sign) * table[pos, None, :, 1].astype(dtype)
    a, b = y[..., first].copy(), y[..., second].copy()
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    return y


def quantise(x, kind):
    """(codes, scales, values) of FP32 vectors, bit for bit."""
    f = np.float32
    bad = ~np.isfinite(x)
    with np.errstate(all="ignore"):
        if kind == "f16":
            h = x.astype(np.float16)
            return h, None, h.astype(f)
        if kind == "int4":
            y = x.reshape(x.shape[:-1] + (-1, 32))
            lo, hi = y.min(-1), y.max(-1)
            sc, low = ((hi - lo) * f(1 / 15)).astype(np.float16), lo.astype(np.float16)
            skip = bad.reshape(y.shape).any(-1) | ~np.isfinite(sc) | ~np.isfinite(low)
            sc, low = np.where(skip, np.float16("nan"), sc), np.where(skip, np.float16("nan"), low)
            inv = np.where(sc > 0, f(1) / sc.astype(f), f(0))
            q = np.clip(np.rint((y - low.astype(f)[..., None]) * inv[..., None]), 0, 15)
            q = np.where(skip[..., None], 0, q)
            v = q.astype(f) * sc.astype(f)[..., None] + low.astype(f)[..., None]
            q = q.astype(np.uint8).reshape(x.shape)
            return q[..., ::2] | q[..., 1::2] << 4, np.stack([sc, low], -1), v.reshape(x.shape)
        top = np.abs(x).max(-1)
        skip = bad.any(-1)
        sc = top * f(1 / (127 if kind == "int8" else 448))
        sc = np.where(sc < f(2.0 ** -120), f(0), sc)
        inv = np.where(sc > 0, f(1) / sc, f(0))
        sc = np.where(skip, f("nan"), sc)
        q = np.where(skip[..., None], f(0), x * inv[..., None])
        if kind == "int8":
            q = np.clip(np.rint(q), -127, 127).astype(np.int8)
            return q, sc, q.astype(f) * sc[..., None]
        q = torch.from_numpy(np.clip(q, -448, 448)).to(torch.float8_e4m3fn)
        return q.view(torch.uint8).numpy(), sc, q.float().numpy() * sc[..., None]


class Pool:
    """A cache with random vectors for every slot of every sequence, and the 64-bit values of all of them."""

    def __init__(self, P, kind, seqs, slots, heads, dim, page, seed=0, spare=2, big=1.0):
        g = gen(seed)
        self.columns = -(-slots // page)
        pages = seqs * self.columns + spare
        self.cache = P.KVCache.empty(pages, page, heads, dim, kind)
        self.table = g.permutation(pages)[: seqs * self.columns].reshape(seqs, self.columns).astype(np.int32)
        self.pages = dev(self.table)
        n = self.columns * page
        self.k = (big * g.standard_normal((seqs, n, heads, dim))).astype(np.float32)
        self.v = g.standard_normal((seqs, n, heads, dim)).astype(np.float32)
        self.kind, self.page = kind, page
        self.write("k", self.k)
        self.write("v", self.v)

    def write(self, x, values, seqs=None, slots=None):
        """Store values (seqs, slots, heads, dim) through numpy, and keep what they stand for."""
        codes, scale, real = quantise(values, self.kind)
        b, n = values.shape[:2]
        seq = np.repeat(np.arange(b) if seqs is None else seqs, n)
        slot = np.tile(np.arange(n) if slots is None else slots, b)
        page, row = dev(self.table[seq, slot // self.page]).long(), dev(slot % self.page).long()
        t = getattr(self.cache, x)
        t = t.view(torch.uint8) if self.kind == "e4m3" else t
        t[page, :, row] = dev(codes.reshape((-1,) + codes.shape[2:]))
        if scale is not None:
            getattr(self.cache, x + "_scale")[page, :, row] = dev(scale.reshape((-1,) + scale.shape[2:]))
        getattr(self, x)[seq, slot] = real.reshape((-1,) + real.shape[2:])


def attention(pool, q, lens, allowed, scale):
    """(out, lse, bound of the error) in 64 bits. allowed (seqs, nodes, nodes): node sees node; None where dead."""
    seqs, nodes, heads, dim = q.shape
    group = heads // pool.k.shape[2]
    out, lse, tol = np.zeros(q.shape), np.full(q.shape[:3], -np.inf), np.zeros(q.shape)
    for b in range(seqs):
        n = lens[b]
        for i in range(nodes):
            sees = np.zeros(pool.k.shape[1], bool)
            if allowed[b, i] is not None:
                sees[:n] = True
                new = allowed[b, i][: max(0, len(sees) - n)]
                sees[n: n + len(new)] = new
            if not sees.any():
                continue
            for h in range(heads):
                k, v = pool.k[b, sees, h // group].astype(float), pool.v[b, sees, h // group].astype(float)
                x = q[b, i, h].astype(float)
                with np.errstate(all="ignore"):
                    s = scale * (k @ x)
                    w = np.exp(s - s.max())
                    out[b, i, h] = (w / w.sum()) @ v
                    lse[b, i, h] = s.max() + math.log(w.sum())
                    a = (w / w.sum()) @ np.abs(v)
                    far = scale * (np.abs(k) @ np.abs(x)).max()
                    four = pool.kind == "int4"
                    ds = (U if four else 0.0) * far + 2 * E * dim * far + 4 * E * np.abs(s).max()
                    tol[b, i, h] = (U * (2 if four else 1) + 2 * ds + 2.0 ** -20) * a
    return out, lse, tol


def check(P, pool, q, lens, mask, counts, allowed, out_dtype=torch.float16, scale=None, want_lse=True, workspace=None):
    seqs, nodes, heads, dim = q.shape
    out = torch.full(q.shape, float("nan"), dtype=out_dtype, device="cuda")
    lse = torch.full(q.shape[:3], float("nan"), dtype=torch.float32, device="cuda") if want_lse else None
    got = pool.cache.tree_attention(dev(q), pool.pages, dev(np.asarray(lens, np.int32)),
                                    mask=None if mask is None else dev(mask),
                                    counts=None if counts is None else dev(np.asarray(counts, np.int32)), scale=scale,
                                    out=out, lse=lse, workspace=workspace)
    assert got is out
    ref, ref_lse, tol = attention(pool, q, np.maximum(lens, 0), allowed, 1 / math.sqrt(dim) if scale is None else scale)
    y = out.double().cpu().numpy()
    if out_dtype == torch.float16:
        tol = tol + U * np.abs(ref) + 2.0 ** -25
    np.testing.assert_array_equal(np.isnan(y), np.isnan(ref))
    ok = np.isfinite(ref)
    worst = np.abs(y[ok] - ref[ok]) - tol[ok]
    assert worst.size == 0 or worst.max() <= 0, worst.max()
    if want_lse:
        z = lse.double().cpu().numpy()
        dead = np.isneginf(ref_lse)
        np.testing.assert_array_equal(np.isneginf(z), dead)
        live = np.isfinite(ref_lse)
        four = pool.kind == "int4"
        far = 64 * U if four else 2.0 ** -10  # scores of these inputs are far below 64
        assert np.all(np.abs(z[live] - ref_lse[live]) <= far)
    return y


def random_tree(g, seqs, nodes):
    parents = np.array([[int(g.integers(max(-1, i - 5), i)) if i else -1 for i in range(nodes)] for _ in range(seqs)],
                       np.int32)
    sees = np.zeros((seqs, nodes, nodes), bool)
    for b in range(seqs):
        for i in range(nodes):
            j = i
            while j >= 0:
                sees[b, i, j] = True
                j = parents[b, j]
    return parents, sees


def words(sees):
    seqs, nodes, _ = sees.shape
    w = np.zeros((seqs, nodes, -(-nodes // 32)), np.uint32)
    for j in range(nodes):
        w[..., j // 32] |= sees[..., j].astype(np.uint32) << np.uint32(j % 32)
    return w.view(np.int32)


def rows_of(sees, counts):
    """attention()'s `allowed`: None for nodes at counts and after; nodes there are not seen."""
    seqs, nodes, _ = sees.shape
    out = np.empty((seqs, nodes), object)
    for b in range(seqs):
        for i in range(nodes):
            out[b, i] = None if i >= counts[b] else sees[b, i] & (np.arange(nodes) < counts[b])
    return out


# -- rope -----------------------------------------------------------------------------


@pytest.mark.parametrize("dim,rot", [(128, 128), (64, 64), (128, 64), (80, 24), (10, 6), (6, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [np.float16, np.float32])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (37, 5)])
def test_rope(P, dim, rot, interleaved, dtype, tokens, heads):
    g = gen(dim + rot + tokens)
    x = g.standard_normal((tokens, heads, dim)).astype(dtype)
    pos = g.integers(0, 50, tokens).astype(np.int32)
    table = table_np(50, rot)
    for sign in (1, -1):
        y = P.rope(dev(x), dev(pos), dev(table), interleaved=interleaved, backward=sign < 0).cpu().numpy()
        ref = rotate(x, pos, table, interleaved, np.float64, sign)
        first, second = pairs(rot, interleaved)
        size = np.abs(x).astype(float)
        size[..., first] = size[..., second] = size[..., first] + size[..., second]
        tol = 3 * E * size + (U * np.abs(ref) + 2.0 ** -25 if dtype == np.float16 else 0)
        assert np.all(np.abs(y - ref) <= tol)
        exact = rotate(x, pos, table, interleaved, np.float32, sign).astype(dtype)
        np.testing.assert_array_equal(y, exact)  # each operation rounded on its own
        np.testing.assert_array_equal(y[..., rot:], x[..., rot:])


def test_rope_gradient(P):
    """backward is the transposed map: against the formula's matrix and against differences of the forward map."""
    g = gen(5)
    tokens, dim, rot = 3, 16, 12
    table, pos = table_np(9, rot) * np.float32(1.25), np.array([0, 4, 8], np.int32)
    for interleaved in (False, True):
        x = g.standard_normal((tokens, 1, dim)).astype(np.float32)
        dy = g.standard_normal((tokens, 1, dim)).astype(np.float32)
        dx = P.rope(dev(dy), dev(pos), dev(table), interleaved=interleaved, backward=True).cpu().numpy()
        f = lambda z: P.rope(dev(z), dev(pos), dev(table), interleaved=interleaved).double().cpu().numpy()  # noqa: E731
        eye = np.eye(dim, dtype=np.float64)
        for tok in range(tokens):
            m = rotate(np.repeat(eye[:, None], 1, 1), np.full(dim, pos[tok]), table, interleaved, np.float64)[:, 0]
            np.testing.assert_allclose(dx[tok, 0], m @ dy[tok, 0].astype(float), rtol=0, atol=16 * E * 8)
        h = np.float32(0.5)  # the map is linear: any step gives its slope
        for e in range(dim):
            up, down = x.copy(), x.copy()
            up[..., e] += h
            down[..., e] -= h
            step = (up[..., e] - down[..., e]).astype(float)
            slope = ((f(up) - f(down)) * dy).sum(-1) / step
            np.testing.assert_allclose(dx[..., e], slope, rtol=0, atol=1e-5)


def test_rope_strides_in_place_and_positions(P):
    g = gen(6)
    big = g.standard_normal((9, 7, 3, 64)).astype(np.float16)
    table = table_np(20, 64)
    pos = np.array([0, 19, 20, -1, 3, 5, 7, 11, 13], np.int32)
    t = dev(big)
    x = t[:, 1:6, 1]  # strided tokens and heads, 128-byte aligned
    with np.errstate(all="ignore"):
        ref = rotate(big[:, 1:6, 1], np.clip(pos, 0, 19), table, False, np.float32).astype(np.float16)
    ref[2:4] = np.nan  # positions outside the table
    y = P.rope(x, dev(pos), dev(table))
    np.testing.assert_array_equal(y.cpu().numpy(), ref)
    assert P.rope(x, dev(pos), dev(table), out=x) is x
    np.testing.assert_array_equal(x.cpu().numpy(), ref)
    keep = np.ones(big.shape, bool)
    keep[:, 1:6, 1] = False
    np.testing.assert_array_equal(t.cpu().numpy()[keep], big[keep])
    odd = dev(g.standard_normal(2 * 3 * 64 + 1).astype(np.float32))[1:].view(2, 3, 64)  # 4-byte aligned
    two = np.array([1, 2], np.int32)
    np.testing.assert_array_equal(P.rope(odd, dev(two), dev(table)).cpu().numpy(),
                                  rotate(odd.cpu().numpy(), two, table, False, np.float32))
    assert P.rope(dev(big[:0, 0]), dev(pos[:0]), dev(table)).shape == (0, 3, 64)


@pytest.mark.parametrize("scaling", [None, "linear", "base", "bands", "ramp"])
def test_rope_table(P, scaling):
    kw = dict(base=500000.0, scaling=scaling, factor=8.0, low=1.0, high=4.0, original=8192.0)
    length, dim = 4096, 128
    freq, att = P.rope_frequencies(dim, **kw)
    t = P.rope_table(length, dim, **kw).double().cpu().numpy()
    angle = np.arange(length)[:, None] * np.array(freq)
    ref = att * np.stack([np.cos(angle), np.sin(angle)], -1)
    # FP64 angles of up to 4096 radians (2^-41 apart), rounded to FP32: half of its spacing there.
    assert np.all(np.abs(t - ref) <= np.spacing(np.abs(ref).astype(np.float32)) / 2.0 + att * 2.0 ** -38)


# -- append and read ---------------------------------------------------------------------


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,rot,interleaved", [(128, 128, False), (64, 64, True), (128, 32, False), (128, 64, True),
                                                 (64, 24, False), (64, 10, True), (128, 0, False)])
@pytest.mark.parametrize("dtype", [np.float16, np.float32])
def test_append_bit_for_bit(P, kind, dim, rot, interleaved, dtype):
    g = gen(dim + rot)
    seqs, heads, q_heads, page, tokens = 3, 2, 5, 16, 23
    cache = P.KVCache.empty(9, page, heads, dim, kind)
    table = g.permutation(9).reshape(seqs, 3).astype(np.int32)
    at = g.permutation(seqs * 48)[:tokens]
    seq, slot = (at // 48).astype(np.int32), (at % 48).astype(np.int32)
    slot[4] = -1  # padding
    k = (g.standard_normal((tokens, heads, dim)) * g.choice([1e-3, 1, 50], (tokens, 1, 1))).astype(dtype)
    v = g.standard_normal((tokens, heads, dim)).astype(dtype)
    k[0] = 0
    v[1, 0, :32] = 0.25  # a group of equal entries
    v[2, 1, 5] = np.inf
    k[3, 0, dim - 1] = np.nan
    q = g.standard_normal((tokens, q_heads, dim)).astype(dtype)
    rope = table_np(48, rot) if rot else None
    pos = np.maximum(slot, 0)
    k_out = torch.empty((tokens, heads, dim), dtype=torch.float16, device="cuda")
    v_out = torch.empty_like(k_out)
    q_out = cache.append(dev(k), dev(v), dev(table), dev(seq), dev(slot), rope=None if rope is None else dev(rope),
                         q=dev(q), interleaved=interleaved, k_out=k_out, v_out=v_out)
    with np.errstate(all="ignore"):
        kr = rotate(k, pos, rope, interleaved, np.float32) if rot else k.astype(np.float32)
        qr = (rotate(q, pos, rope, interleaved, np.float32) if rot else q.astype(np.float32)).astype(np.float16)
    qr[4] = 0
    np.testing.assert_array_equal(q_out.cpu().numpy(), qr)
    for x, y, got in (("k", kr, k_out), ("v", v.astype(np.float32), v_out)):
        codes, scale, real = quantise(y, kind)
        want = np.zeros(tuple(cache.k.shape[:3]) + codes.shape[2:], codes.dtype)
        put = [i for i in range(tokens) if slot[i] >= 0]
        for i in put:
            want[table[seq[i], slot[i] // page], :, slot[i] % page] = codes[i]
        have = getattr(cache, x)
        have = (have.view(torch.uint8) if kind == "e4m3" else have).cpu().numpy()
        np.testing.assert_array_equal(have, want)
        if scale is not None:
            want = np.zeros(tuple(cache.k.shape[:3]) + scale.shape[2:], scale.dtype)
            for i in put:
                want[table[seq[i], slot[i] // page], :, slot[i] % page] = scale[i]
            np.testing.assert_array_equal(getattr(cache, x + "_scale").cpu().numpy(), want)
        with np.errstate(all="ignore"):
            real = real.astype(np.float16)
        real[4] = 0
        np.testing.assert_array_equal(got.cpu().numpy(), real)


def test_append_strides_positions_and_bounds(P):
    g = gen(8)
    cache = P.KVCache.empty(4, 16, 2, 64, "int8")
    table = np.array([[0, 7], [2, -1]], np.int32)  # page 7 and -1 do not exist
    qkv = g.standard_normal((6, 2 * 64 * 4)).astype(np.float16)  # q | k | v of each token in one row
    t = dev(qkv)
    q, k, v = t[:, :256].view(6, 4, 64), t[:, 256:384].view(6, 2, 64), t[:, 384:].view(6, 2, 64)
    seq = np.array([0, 1, 0, 1, 2, -1], np.int32)
    slot = np.array([3, 15, 16, 31, 0, 0], np.int32)  # two in pages that do not exist, two of no sequence
    pos = np.array([5, 0, 1, 2, 3, 4], np.int32)
    rope = table_np(6, 64)
    cache.append(k, v, dev(table), dev(seq), dev(slot), rope=dev(rope), positions=dev(pos), q=q, q_out=q)
    n = lambda x, a: rotate(qkv[:, x: x + a * 64].reshape(6, a, 64), pos, rope, False, np.float32)  # noqa: E731
    np.testing.assert_array_equal(q.cpu().numpy(), n(0, 4).astype(np.float16))
    codes = quantise(n(256, 2), "int8")[0]
    want = np.zeros((4, 2, 16, 64), np.int8)
    want[0, :, 3], want[2, :, 15] = codes[0], codes[1]
    np.testing.assert_array_equal(cache.k.cpu().numpy(), want)
    cache.append(k[:0], v[:0], dev(table), dev(seq[:0]), dev(slot[:0]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (128, 256)])
def test_read(P, kind, dim, page):
    pool = Pool(P, kind, 3, 300, 2, dim, page, seed=dim + page)
    pool.k[1, 7] *= 1  # the values that the codes stand for
    lens = np.array([300, 0, 131], np.int32)
    for dtype in (torch.float16, torch.float32):
        for first, count in ((0, 300), (5, 1), (130, 77), (299, 0), (290, 400)):
            k, v = pool.cache.read(pool.pages, dev(lens), first=first, count=count, dtype=dtype)
            for got, x in ((k, pool.k), (v, pool.v)):
                want = np.zeros((3, count, 2, dim), np.float32)
                for b in range(3):
                    n = min(max(lens[b] - first, 0), count)
                    want[b, :n] = x[b, first: first + n]
                want = want.astype(np.float16) if dtype == torch.float16 else want
                if kind == "int4" and dtype == torch.float16:  # one rounding there, two in numpy
                    assert np.all(np.abs(got.cpu().numpy().astype(float) - want) <= 2 * U * np.abs(want) + 2.0 ** -24)
                elif kind == "int4":
                    assert np.all(np.abs(got.cpu().numpy() - want) <= 2.0 ** -23 * (np.abs(want) + 8))
                else:
                    np.testing.assert_array_equal(got.cpu().numpy(), want)
    pool.table[0, 0], pool.table[2, 0] = -1, 10 ** 6  # pages that do not exist read as zeros
    k, _ = pool.cache.read(dev(pool.table), dev(lens), count=page)
    assert not k[0].any() and not k[2].any()


# -- tree attention -----------------------------------------------------------------------


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes,group,page", [(1, 1, 16), (1, 4, 64), (3, 5, 32), (7, 4, 16), (16, 4, 128), (33, 3, 16),
                                              (64, 8, 64), (20, 16, 256)])
def test_tree(P, kind, dim, nodes, group, page):
    g = gen(nodes * group + dim)
    seqs, heads = 4, 2
    lens = np.array([131, 0, 1, 517], np.int32)
    pool = Pool(P, kind, seqs, 517 + nodes, heads, dim, page, seed=nodes + dim)
    parents, sees = random_tree(g, seqs, nodes)
    counts = np.array([nodes, max(1, nodes // 2), 0, nodes], np.int32)
    q = (1.5 * g.standard_normal((seqs, nodes, heads * group, dim))).astype(np.float16)
    mask = words(sees)
    np.testing.assert_array_equal(P.tree_mask(dev(parents)).cpu().numpy(), mask)
    check(P, pool, q, lens, mask, counts, rows_of(sees, counts))
    check(P, pool, q, lens, None, None, rows_of(np.tril(np.ones((seqs, nodes, nodes), bool)), [nodes] * seqs),
          out_dtype=torch.float32)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("length", [1, 15, 16, 17, 31, 33, 127, 129, 255, 257, 1023, 4099])
def test_one_token_lengths(P, kind, length):
    g = gen(length)
    pool = Pool(P, kind, 2, length + 1, 1, 128, 16, seed=length)
    q = g.standard_normal((2, 1, 4, 128)).astype(np.float16)
    lens = np.array([length, length // 2], np.int32)
    check(P, pool, q, lens, None, None, rows_of(np.ones((2, 1, 1), bool), [1, 1]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nodes", [1, 16])
def test_long_and_ragged(P, kind, nodes):
    """Items that span several CTAs beside items that do not."""
    g = gen(3)
    lens = np.array([9001, 17, 0, 2500, 64, 1], np.int32)
    pool = Pool(P, kind, 6, 9001 + nodes, 1, 64, 64, seed=11)
    q = g.standard_normal((6, nodes, 2, 64)).astype(np.float16)
    _, sees = random_tree(g, 6, nodes)
    a = check(P, pool, q, lens, words(sees), None, rows_of(sees, [nodes] * 6))
    b = check(P, pool, q, lens, words(sees), None, rows_of(sees, [nodes] * 6))
    np.testing.assert_array_equal(a, b)  # the order of the sums does not depend on timing


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (128, 256)])
def test_many_rows_long_runs(P, kind, dim, page):
    """The tensor-core kernel: long items, short and empty ones, several runs to a CTA, rows beyond one block."""
    g = gen(dim + page)
    seqs, nodes, group = 24, 35, 4  # 140 rows
    lens = g.integers(0, 700, seqs).astype(np.int32)
    lens[[0, 5, 9]] = 6500, 0, 4099
    pool = Pool(P, kind, seqs, 6500 + nodes, 1, dim, page, seed=7)
    q = (1.5 * g.standard_normal((seqs, nodes, group, dim))).astype(np.float16)
    _, sees = random_tree(g, seqs, nodes)
    counts = g.integers(0, nodes + 1, seqs).astype(np.int32)
    workspace = pool.cache.make_workspace(dev(q))
    a = check(P, pool, q, lens, words(sees), counts, rows_of(sees, counts), workspace=workspace)
    for _ in range(3):  # the order of the sums does not depend on timing
        b = pool.cache.tree_attention(dev(q), pool.pages, dev(lens), mask=dev(words(sees)), counts=dev(counts),
                                      workspace=workspace)
        np.testing.assert_array_equal(a, b.double().cpu().numpy())
    P.workspace_status(workspace)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nodes,group", [(6, 2), (40, 4)])
def test_masked_places_hold_nan_and_infinity(P, kind, nodes, group):
    """Slots after a sequence's end, and nodes that a node does not see."""
    g = gen(9)
    lens = np.array([40, 0, 130], np.int32)
    pool = Pool(P, kind, 3, 256, 2, 128, 16, seed=4)
    bad = np.full((1, 1, 2, 128), np.nan, np.float32)
    for b in range(3):  # nothing after the nodes may matter, whatever is there
        for at in range(lens[b] + nodes, 256):
            pool.write("k", bad, [b], [at])
            pool.write("v", bad * (1 if at % 2 else np.inf), [b], [at])
    sees = np.zeros((3, nodes, nodes), bool)
    sees[:, np.arange(nodes), np.arange(nodes)] = True
    sees[:, :, 0] = True
    sees[:, 3] = False  # a node that sees the cached tokens alone, and in sequence 1 nothing
    pool.write("v", bad, [0], [lens[0] + 2])  # node 2, which only node 2 sees
    pool.write("k", bad, [1], [lens[1] + 4])
    inf = g.standard_normal((1, 1, 2, 128)).astype(np.float32)
    inf[..., 7] = np.inf
    pool.write("v", inf, [2], [lens[2] + 1])
    q = g.standard_normal((3, nodes, 2 * group, 128)).astype(np.float16)
    y = check(P, pool, q, lens, words(sees), None, rows_of(sees, [nodes] * 3), want_lse=False)
    assert np.isnan(y[0, 2]).all() and not np.isnan(y[0, [0, 1, 3, 4, 5]]).any()
    assert np.isnan(y[1, 4]).all() and not y[1, 3].any()
    assert not np.isfinite(y[2, 1, :, 7]).any() and np.isfinite(y[2, 0]).all()


def exact_attention(pool, q, lens, scale):
    """Causal attention of the nodes in 64 bits, as tensors on the GPU."""
    k, v, x = (torch.from_numpy(t).cuda().double() for t in (pool.k, pool.v, q))
    seqs, nodes, heads, _ = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    for b in range(seqs):
        n = int(lens[b]) + nodes
        hide = torch.ones((nodes, n), dtype=torch.bool, device="cuda").triu(1 + int(lens[b]))
        for h in range(heads):
            e = scale * (x[b, :, h] @ k[b, :n, h * k.shape[2] // heads].T)
            out[b, :, h] = torch.softmax(e.masked_fill(hide, -math.inf), -1) @ v[b, :n, h * k.shape[2] // heads]
    return out


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes", [3, 40, 64])
@pytest.mark.parametrize("big", [1.0, 600.0, -2.0])
def test_four_bit_keys_are_exact(P, dim, nodes, big):
    """Scores of INT4 keys take the scale, low and code of each group as they are, whichever kernel a call takes.

    What is left are the roundings to FP16 of each weight and each value, both of at most U and independent: of sums of
    random terms sqrt(2 / 3) U of the norm. Rounded keys, with a few channels of six times the others, make that twice
    as much. Queries of 600 have sums over a group that are beyond FP16; the scale undoes them."""
    g = gen(16 + nodes)
    pool = Pool(P, "int4", 1, 4000 + nodes, 2, dim, 64, seed=9)
    k = pool.k * np.where(g.random((1, 1, 2, dim)) < 0.05, 6, 1).astype(np.float32)
    k[..., :32] += 3  # a group off zero
    pool.write("k", k)
    q = (1.5 * g.standard_normal((1, nodes, 8, dim))).astype(np.float32)
    if big == 600.0:
        q = np.abs(q)  # sums of 32 entries above 8192, FP16 ends at 65504
    q = (abs(big) * q).astype(np.float16)
    scale = dim ** -0.5 / big
    lens = np.array([4000], np.int32)
    out = pool.cache.tree_attention(dev(q), pool.pages, dev(lens), scale=scale, out=torch.empty(q.shape, device="cuda"))
    want = exact_attention(pool, q, lens, scale)
    assert (out - want).norm() <= U * want.norm(), float((out - want).norm() / want.norm())


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("nodes", [3, 20])
def test_a_large_weight_counts_as_it_is_rounded(P, dim, nodes):
    """INT4: one key has nearly all of the weight, and its value no rounding of its own.

    The weight is off by up to 2^-12 of itself, in the sum and in the divisor, so that of 120 to 250 times the others'
    weight 2^-12 / 100 is left, as of the others. Taken for what it was before rounding, it leaves 2^-12."""
    g = gen(17)
    seqs, heads = 40, 8  # more items than the GPU has SMs: many of them stay whole
    pool = Pool(P, "int4", seqs, 384, heads, dim, 64, seed=4)
    k, v = np.full((seqs, 384, heads, dim), -1, np.float32), np.zeros((seqs, 384, heads, dim), np.float32)
    k[:, 0], k[:, 130] = 0, 0.5  # a group of equal entries is its low: no code, no rounding
    v[:, 130] = np.float16(0.7)
    pool.write("k", k)
    pool.write("v", v)
    # Scores ln 120 to ln 250 above the first keys' largest, 0: below the 2^8 that move the reference.
    want = np.log(g.uniform(120, 250, (seqs, nodes, heads)))
    q = np.repeat((want / (0.5 * dim ** 0.5))[..., None], dim, -1).astype(np.float16)
    lens = np.full(seqs, 340, np.int32)
    out = pool.cache.tree_attention(dev(q), pool.pages, dev(lens), out=torch.empty(q.shape, device="cuda"))
    ref = exact_attention(pool, q, lens, dim ** -0.5)
    assert ((out - ref).abs() <= 2.0 ** -17 * ref.abs()).all(), float(((out - ref) / ref).abs().max())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nodes", [4, 40])
def test_nan_values_of_the_least_weight(P, kind, nodes):
    """A node's NaN or infinite value whose weight is e^-362: it still reaches the rows that see it, and no other."""
    g = gen(15)
    pool = Pool(P, kind, 2, 100, 1, 128, 16, seed=4)
    lens = np.array([50, 35], np.int32)
    odd = g.standard_normal((1, 1, 1, 128)).astype(np.float32)
    odd[..., 9] = np.nan
    for b in range(2):
        pool.write("k", np.full((1, 1, 1, 128), -8, np.float32), [b], [lens[b] + 1])
        pool.write("v", odd, [b], [lens[b] + 1])
        odd[..., 9] = np.inf
    q = np.full((2, nodes, 1, 128), 4, np.float16)
    sees = np.repeat(np.tril(np.ones((nodes, nodes), bool))[None], 2, 0)
    sees[:, 2:, 1] = False  # node 1 sees itself; so does one node more
    sees[:, 3, 1] = True
    y = check(P, pool, q, lens, words(sees), None, rows_of(sees, [nodes] * 2), want_lse=False)
    assert not np.isfinite(y[:, [1, 3], 0, 9]).any() and np.isfinite(np.delete(y, [1, 3], 1)).all()


@pytest.mark.parametrize("kind", ["f16", "int8"])
@pytest.mark.parametrize("nodes", [5, 33])
def test_infinite_values_among_empty_sequences(P, kind, nodes):
    """Many sequences to a CTA, most of them empty: each one's odd values are its own."""
    g, seqs = gen(12), 1024
    pool = Pool(P, kind, seqs, 48, 1, 64, 16, seed=6)
    inf = g.standard_normal((1, 1, 1, 64)).astype(np.float32)
    inf[..., 7] = np.inf
    for b in range(4, seqs, 8):
        pool.write("v", inf, [b], [0])
    counts = np.where(np.arange(seqs) % 4 == 0, nodes, 0)
    sees = np.repeat(np.eye(nodes, dtype=bool)[None], seqs, 0)
    q = g.standard_normal((seqs, nodes, 1, 64)).astype(np.float16)
    y = check(P, pool, q, np.zeros(seqs, np.int32), words(sees), counts, rows_of(sees, counts))
    assert not np.isfinite(y[4::8, 0, :, 7]).any() and np.isfinite(y[0::8]).all() and np.isfinite(y[4::8, 1:]).all()


def test_missing_pages_strides_masks_and_scales(P):
    g = gen(10)
    nodes, group, dim = 5, 3, 128
    pool = Pool(P, "int8", 3, 200, 2, dim, 16, seed=2)
    lens = np.array([100, 150, 195], np.int32)
    _, sees = random_tree(g, 1, nodes)
    q = g.standard_normal((3, nodes, 6, dim)).astype(np.float16)
    allowed = rows_of(np.repeat(sees, 3, 0), [nodes] * 3)
    check(P, pool, q, lens, words(sees), None, allowed, scale=0.3)  # one mask for all sequences
    # Strided queries and outputs.
    wide_q, wide_o = dev(np.zeros((3, nodes, 6, 256), np.float16)), torch.zeros((nodes, 3, 6, 136), device="cuda")
    wide_q[..., 128:] = dev(q)
    out = wide_o.transpose(0, 1)[..., :128]
    pool.cache.tree_attention(wide_q[..., 128:], pool.pages, dev(lens), mask=dev(words(sees)), out=out)
    ref, _, tol = attention(pool, q, lens, allowed, dim ** -0.5)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= tol)
    assert not wide_o[..., 128:].any()
    # Pages that do not exist are not seen.
    gone = pool.table.copy()
    gone[1, 2], gone[2, 12], gone[0, 0] = -1, 10 ** 6, -5
    out = pool.cache.tree_attention(dev(q), dev(gone), dev(lens), mask=dev(words(sees)), out=torch.empty(
        q.shape, device="cuda"))
    for b, col in ((1, 2), (2, 12), (0, 0)):
        keep = np.ones(pool.k.shape[1], bool)
        keep[16 * col: 16 * col + 16] = False
        for i in range(nodes):
            see = keep.copy()
            see[lens[b]:] = False
            see[lens[b]: lens[b] + nodes] = sees[0, i] & keep[lens[b]: lens[b] + nodes]
            for h in range(6):
                s = pool.k[b, see, h // 3].astype(float) @ q[b, i, h].astype(float) * dim ** -0.5
                w = np.exp(s - s.max())
                v = pool.v[b, see, h // 3].astype(float)
                got = out[b, i, h].double().cpu().numpy()
                assert np.all(np.abs(got - w @ v / w.sum()) <= (U + 1e-4) * (w @ np.abs(v)) / w.sum())
    # Slots beyond the table are not there; negative lengths are 0.
    short = np.array([208, 206, -3], np.int32)
    check(P, pool, q, short, words(sees), None, allowed)


def test_workspace_serves_other_shapes_streams_and_graphs(P):
    g = gen(12)
    pool = Pool(P, "int8", 4, 3000, 2, 64, 64, seed=5)
    big = torch.zeros(pool.cache.workspace_bytes(4, 64, 16), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for nodes, group, lens in ((1, 2, [2900, 5, 0, 1000]), (40, 8, [2900, 5, 0, 1000]), (2, 1, [1, 2, 3, 4]),
                               (9, 3, [2000, 0, 2999, 700])):
        lens = np.minimum(np.array(lens, np.int32), 3000 - nodes)
        q = g.standard_normal((4, nodes, 2 * group, 64)).astype(np.float16)
        _, sees = random_tree(g, 4, nodes)
        check(P, pool, q, lens, words(sees), None, rows_of(sees, [nodes] * 4), workspace=big)
        tq, tl, tm = dev(q), dev(lens), dev(words(sees))
        plain = pool.cache.tree_attention(tq, pool.pages, tl, mask=tm, workspace=big)
        side.wait_stream(torch.cuda.current_stream())
        other = pool.cache.tree_attention(tq, pool.pages, tl, mask=tm, stream=side)
        side.synchronize()
        assert torch.equal(plain, other)
        out = torch.zeros_like(plain)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pool.cache.tree_attention(tq, pool.pages, tl, mask=tm, out=out, workspace=big)
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(plain, out)
    P.workspace_status(big)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nodes,dim", [(2, 64), (2, 128), (40, 64), (40, 128)])
def test_waits_that_give_up(P, kind, nodes, dim):
    """A budget of one cycle, which waits for copies do not keep: the calls end and say so, the arrival counters are at
    zero again, and the next calls on the cleared workspace give what they gave before."""
    torch.manual_seed(14)
    cache = P.KVCache.empty(400, 256, 8, dim, kind)  # enough to keep the memory busy
    for t in (cache.k, cache.v):
        if kind == "f16":
            t.normal_()
        else:  # E4M3: no NaN, at most 30
            t.view(torch.uint8).random_().bitwise_and_(0xCF if kind == "e4m3" else 0xFF)
    for t in (cache.k_scale, cache.v_scale):
        if t is not None:
            t.uniform_(0.001, 0.01)
    pages = torch.randperm(400, device="cuda").to(torch.int32).view(16, 25)
    lens = torch.randint(0, 6300, (16,), device="cuda").to(torch.int32)
    q = torch.randn((16, nodes, 32, dim), device="cuda").half()
    workspace = cache.make_workspace(q)
    run = lambda: cache.tree_attention(q, pages, lens, workspace=workspace)  # noqa: E731
    before = run()
    P.workspace_status(workspace)
    sweep = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")  # twice the L2: copies come from the memory
    old = P.get_wait_cycles()
    try:
        P.set_wait_cycles(1)
        for _ in range(40):
            sweep.zero_()
            run()
        torch.cuda.synchronize()
    finally:
        P.set_wait_cycles(old)
    with pytest.raises(P.AF1Error) as e:
        P.workspace_status(workspace)
    assert e.value.code == -7
    assert not workspace[256:4352].any()
    workspace.zero_()
    for _ in range(3):
        assert torch.equal(run(), before)
    P.workspace_status(workspace)


@pytest.mark.parametrize("nodes,group", [(1, 4), (40, 4)])
def test_default_workspace_clears_its_head_alone(P, nodes, group):
    """What a workspace holds behind its head may be anything, and is left as it is."""
    cache = P.KVCache.empty(8, 64, 2, 64, "f16")
    cache.k.normal_(), cache.v.normal_()
    q = torch.randn((1, nodes, 2 * group, 64), device="cuda").half()
    size, head = cache.workspace_bytes(1, nodes, 2 * group), 65792
    old = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    at = old.data_ptr()
    del old
    workspace = cache.make_workspace(q)
    assert not workspace[:head].any()
    if workspace.data_ptr() == at:  # the allocator gave the same memory
        assert workspace[head:].eq(255).all()
    else:
        workspace[head:] = 255
    pages, lens = torch.arange(8, device="cuda").to(torch.int32)[None], torch.tensor([500 - nodes], dtype=torch.int32,
                                                                                     device="cuda")
    with pytest.raises(P.AF1Error) as e:  # leaves no error behind
        cache.tree_attention(q.cpu(), pages, lens)
    assert e.value.code == -2 and not cache.make_workspace(q.cpu()).any()
    zeros = torch.zeros(size, dtype=torch.uint8, device="cuda")
    a = cache.tree_attention(q, pages, lens, workspace=workspace)
    assert torch.equal(a, cache.tree_attention(q, pages, lens, workspace=zeros))
    assert torch.equal(a, cache.tree_attention(q, pages, lens))
    assert not workspace[:head].any() and not zeros[:head].any()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nodes", [1, 40])
def test_largest_scale(P, kind, nodes):
    """Scores of 0 stay 0 at the largest scale; larger ones, whose multiple by log2(e) is infinite, are refused."""
    pool = Pool(P, kind, 2, 100, 1, 64, 16, seed=1)
    q = np.zeros((2, nodes, 1, 64), np.float16)
    sees = np.repeat(np.tril(np.ones((nodes, nodes), bool))[None], 2, 0)
    lens = np.array([60, 7], np.int32)
    for scale in (1e30, -1e30, 0.0):
        check(P, pool, q, lens, None, None, rows_of(sees, [nodes] * 2), scale=scale)
    for scale in (3e38, -3e38):
        with pytest.raises(P.AF1Error) as e:
            pool.cache.tree_attention(dev(q), pool.pages, dev(lens), scale=scale)
        assert e.value.code == -1


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nodes,group", [(5, 3), (40, 4)])  # either kernel
@pytest.mark.parametrize("page", [16, 64, 256])
def test_forms_of_both_kernels(P, kind, nodes, group, page):
    """One mask for all sequences, scales of either sign and 0, strided queries and outputs, pages that do not exist (in
    the prefix, below nodes, a whole tile of keys), slots beyond the table, negative lengths."""
    g = gen(nodes + page)
    seqs, heads, dim = 3, 2, 128
    pool = Pool(P, kind, seqs, 700, heads, dim, page, seed=3)
    slots = pool.columns * page
    lens = np.array([300, 513, 640], np.int32)
    _, sees = random_tree(g, 1, nodes)
    mask = words(sees)
    q = g.standard_normal((seqs, nodes, heads * group, dim)).astype(np.float16)
    allowed = rows_of(np.repeat(sees, seqs, 0), [nodes] * seqs)
    check(P, pool, q, lens, mask, None, allowed, scale=0.3)
    check(P, pool, q, lens, mask, None, allowed, scale=0.0)
    # A negative scale is the positive one of the opposite queries.
    want, _, tol = attention(pool, -q, lens, allowed, 0.2)
    out = pool.cache.tree_attention(dev(q), pool.pages, dev(lens), mask=dev(mask), scale=-0.2,
                                    out=torch.empty(q.shape, device="cuda"))
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)
    # Strided queries and outputs.
    ref, ref_lse, tol = attention(pool, q, lens, allowed, dim ** -0.5)
    wide_q, wide_o = dev(np.zeros((seqs, nodes, heads * group, 256), np.float16)), torch.zeros(
        (nodes, seqs, heads * group, 136), device="cuda")
    wide_q[..., 128:] = dev(q)
    out = wide_o.transpose(0, 1)[..., :128]
    pool.cache.tree_attention(wide_q[..., 128:], pool.pages, dev(lens), mask=dev(mask), out=out)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= tol)
    assert not wide_o[..., 128:].any()
    # Pages that do not exist: what is there is as if it were outside every mask.
    gone = pool.table.copy()
    keep = np.ones((seqs, slots), bool)
    lost = [(0, 0), (0, 290 // page), (1, 513 // page), (2, 128 // page), (2, 255 // page), (2, 655 // page)]
    for n, (b, col) in enumerate(lost):
        gone[b, col] = (-1, 10 ** 6, -(2 ** 31))[n % 3]
        keep[b, page * col: page * col + page] = False
    out = pool.cache.tree_attention(dev(q), dev(gone), dev(lens), mask=dev(mask), out=torch.empty(q.shape, device="cuda"))
    for b in range(seqs):
        for i in range(nodes):
            see = keep[b].copy()
            see[lens[b]:] = False
            new = sees[0, i][: slots - lens[b]]
            see[lens[b]: lens[b] + nodes][: len(new)] = new & keep[b, lens[b]: lens[b] + nodes]
            for h in range(heads * group):
                k, v = pool.k[b, see, h // group].astype(float), pool.v[b, see, h // group].astype(float)
                x = q[b, i, h].astype(float)
                e = k @ x * dim ** -0.5
                w = np.exp(e - e.max()) if e.size else e
                want = w @ v / w.sum() if e.size else np.zeros(dim)
                four = kind == "int4"
                far = dim ** -0.5 * (np.abs(k) @ np.abs(x)).max() if e.size else 0.0
                ds = (U if four else 0.0) * far + 2 * E * dim * far + 4 * E * np.abs(e).max(initial=0)
                a = w @ np.abs(v) / w.sum() if e.size else np.zeros(dim)
                assert np.all(np.abs(out[b, i, h].double().cpu().numpy() - want) <=
                              (U * (2 if four else 1) + 2 * ds + 2.0 ** -20) * a)
    # Slots beyond the table are not there; negative lengths are 0.
    short = np.array([slots, slots - 2, -3], np.int32)
    check(P, pool, q, short, mask, None, allowed)


def test_stream_handles(P, monkeypatch):
    """The current stream, also without torch's private functions."""
    from paper_2609_06161_gb300 import attention as A
    side = torch.cuda.Stream()
    for missing in ((), ("_raw_stream",), ("_raw_stream", "_raw_device")):
        for name in missing:
            monkeypatch.setattr(A, name, None)
        assert A._stream_handle(None) == torch.cuda.current_stream().cuda_stream
        assert A._stream_handle(side) == side.cuda_stream
        with torch.cuda.stream(side):
            assert A._stream_handle(None) == side.cuda_stream


def test_limits_of_sequences_nodes_and_heads(P):
    """The largest of what the header allows, and the next."""
    cache = P.KVCache.empty(1, 16, 1, 64, "int8")

    def call(sequences=1, nodes=1, heads=1):
        q = torch.zeros((sequences, nodes, heads, 64), dtype=torch.float16, device="cuda")
        return cache.tree_attention(q, torch.zeros((sequences, 1), dtype=torch.int32, device="cuda"),
                                    torch.zeros(sequences, dtype=torch.int32, device="cuda"))
    assert not any(call(**most).any() for most in (dict(sequences=1024), dict(nodes=64), dict(heads=65536)))
    for bad in (dict(sequences=1025), dict(nodes=65), dict(heads=65537)):
        with pytest.raises(P.AF1Error) as e:
            call(**bad)
        assert e.value.code == -1


def test_workspace_checks_the_table(P):
    cache = P.KVCache.empty(4, 16, 2, 64, "int8")
    q, table = torch.zeros((2, 3, 4, 64), dtype=torch.float16, device="cuda"), torch.zeros((2, 2), device="cuda")
    assert cache.make_workspace(q, table.int()).numel() == cache.make_workspace(q).numel()
    for bad in (table, table.int()[:1], table.int()[0], table.int().t()):
        with pytest.raises(ValueError):
            cache.make_workspace(q, bad)


def test_offsets_past_32_bits(P):
    """A cache of more than 2^32 bytes and 2^31 entries: its last pages."""
    g = gen(13)
    pages, page, heads, dim = 20000, 256, 8, 128
    cache = P.KVCache.empty(pages, page, heads, dim, "int8")
    assert cache.k.numel() > 2 ** 32
    table = np.array([[pages - 1, 0], [1, pages - 2]], np.int32)
    n = 2 * 300
    seq, slot = np.repeat([0, 1], 300).astype(np.int32), np.tile(np.arange(300), 2).astype(np.int32)
    k, v = (g.standard_normal((n, heads, dim)).astype(np.float16) for _ in "kv")
    cache.append(dev(k), dev(v), dev(table), dev(seq), dev(slot))
    lens = np.array([299, 299], np.int32)
    rk, rv = cache.read(dev(table), dev(lens + 1), count=300, dtype=torch.float32)
    pool = type("Pool", (), {})()
    pool.kind, pool.cache, pool.pages = "int8", cache, dev(table)
    pool.k, pool.v = (quantise(x.astype(np.float32), "int8")[2].reshape(2, 300, heads, dim) for x in (k, v))
    np.testing.assert_array_equal(rk.cpu().numpy(), pool.k)
    np.testing.assert_array_equal(rv.cpu().numpy(), pool.v)
    q = g.standard_normal((2, 1, heads, dim)).astype(np.float16)
    check(P, pool, q, lens, None, None, rows_of(np.ones((2, 1, 1), bool), [1, 1]))


# -- scores -----------------------------------------------------------------------------------


def score_check(P, x, tokens, top, temperature=1.0):
    """x: a CUDA tensor (rows, vocab), perhaps strided."""
    got = P.token_logprobs(x, None if tokens is None else dev(tokens), top=top, temperature=temperature)
    lp, ent = got[0].double().cpu().numpy(), got[1].double().cpu().numpy()
    y = x.double().cpu().numpy()
    z = y / temperature
    with np.errstate(all="ignore"):
        m = z.max(-1, keepdims=True)
        d = np.where(np.isneginf(z), -np.inf, z - np.where(np.isneginf(m), 0, m))
        lse = np.log(np.exp(d).sum(-1, keepdims=True))  # less the maximum
        ref = np.where(np.isneginf(z), np.where(np.isnan(lse), np.nan, -np.inf), d - lse)
        p = np.exp(ref)
        h = -np.where(p > 0, p * ref, np.where(np.isnan(p), np.nan, 0)).sum(-1)
    # FP32 sums of vocab / 256 entries to a thread at least, each exponent off by its argument's rounding.
    vocab = x.shape[1]
    base = E * (vocab / 256 + 128)

    def near(a, b, slack):
        np.testing.assert_array_equal(np.isnan(a), np.isnan(b))
        np.testing.assert_array_equal(np.isneginf(a), np.isneginf(b))
        ok = np.isfinite(b)
        assert np.all(np.abs(a[ok] - b[ok]) <= base + slack * E * (1 + np.abs(b[ok])))

    if tokens is not None:
        inside = (tokens >= 0) & (tokens < vocab)
        want = np.take_along_axis(ref, np.clip(tokens, 0, vocab - 1), -1)
        want = np.where(inside, want, np.where(np.isnan(lse), np.nan, -np.inf))
        near(lp, want, 8)
    # Entropy sums p log p: errors of the logarithms (up to 100 here) by their weights.
    np.testing.assert_array_equal(np.isnan(ent), np.isnan(h))
    ok = np.isfinite(h)
    assert np.all(np.abs(ent[ok] - h[ok]) <= base * (2 + np.abs(h[ok])) + 64 * E * (1 + np.abs(h[ok])))
    if top:
        order = np.where(np.isnan(y), np.inf, y)
        nan_first = np.isnan(y)
        ids = np.lexsort((np.broadcast_to(np.arange(vocab), y.shape), -order, ~nan_first), axis=-1)[:, :top]
        np.testing.assert_array_equal(got[3].cpu().numpy(), ids)
        near(got[2].double().cpu().numpy(), np.take_along_axis(ref, ids, -1), 8)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (1, 7, 7), (3, 33, 32), (2, 255, 5), (5, 1000, 20), (7, 4099, 32),
                                            (2, 32000, 8), (1, 128001, 20), (700, 513, 3), (3, 5000, 0)])
def test_scores(P, dtype, rows, vocab, top):
    g = gen(rows + vocab)
    x = dev((3 * g.standard_normal((rows, vocab))).astype(np.float32)).to(dtype)
    tokens = g.integers(-1, vocab + 1, (rows, 3)).astype(np.int32)
    score_check(P, x, tokens, top)
    score_check(P, x, tokens[:, :1], top, temperature=0.5)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_scores_of_hard_rows(P, dtype):
    g = gen(20)
    vocab, low = 3001, torch.finfo(dtype).min
    x = torch.zeros((13, vocab), dtype=dtype, device="cuda")  # row 0: all equal
    r = dev(g.standard_normal((13, vocab)).astype(np.float32)).to(dtype)
    x[1] = torch.arange(vocab, device="cuda").to(dtype) / 256  # ascending
    x[2] = -x[1]
    x[3] = float("-inf")  # nothing allowed
    x[4] = float("-inf")
    x[4, 2999] = 3.0  # one allowed
    x[5] = torch.where(r[5] < 0, float("-inf"), r[5])
    x[6] = torch.where(r[6] < 1, low, r[6])  # banned by the lowest value
    x[7] = low
    x[8] = r[8]
    x[8, 17] = float("nan")
    x[9] = r[9]
    x[9, 2000] = float("inf")
    x[10] = torch.round(r[10])  # many ties
    x[11, ::2] = -0.0  # equal to 0
    x[12] = 60 * r[12]
    tokens = np.stack([g.permutation(vocab)[:4] for _ in range(13)]).astype(np.int32)
    tokens[:, 0] = 2999
    score_check(P, x, tokens, 32)
    score_check(P, x, None, 0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_scores_of_long_rows(P, dtype):
    """Rows that a thread passes over in several stretches, the largest entries in any of them."""
    g, vocab = gen(22), 2200003
    up = torch.arange(vocab, device="cuda") / 131072
    r = dev(g.standard_normal((4, vocab)).astype(np.float32))
    r[1, -5], r[2, : 20], r[2, 1500000:1500009] = float("nan"), 30.0, 30.0
    x = torch.stack([up, -up, torch.zeros_like(up), *r]).to(dtype)
    tokens = g.integers(0, vocab, (7, 2)).astype(np.int32)
    score_check(P, x, tokens, 32)
    score_check(P, x[3:], tokens[3:], 1)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("temperature", [1e-30, 1e-10, 1e-8, 1e-6, 1e-4, 1e-2, 30.0, 1e30])
def test_scores_at_any_temperature(P, dtype, temperature):
    """The largest entry before the first 16-byte boundary, after the last one, and between; rows that are all ends."""
    g = gen(23)
    for vocab in (5, 33, 4099, 40003):
        for first in (0, 3):
            big = dev((3 * g.standard_normal((6, vocab + 11))).astype(np.float32)).to(dtype)
            x = big[:, first: first + vocab]
            at = [0, vocab - 1, vocab // 2, 1, max(0, vocab - 3), vocab // 3]
            x[torch.arange(6), torch.tensor(at)] = 17.36
            x[5, at[4]] = 17.36  # equal entries, one of them in an end
            x[0, 2] = 17.34375  # next to the largest
            tokens = g.integers(0, vocab, (6, 3)).astype(np.int32)
            tokens[:, 0] = at
            # The library is given the temperature in FP32.
            score_check(P, x, tokens, min(vocab, 9), temperature=float(np.float32(temperature)))


def test_scores_strides(P):
    g = gen(21)
    for dtype in (torch.float16, torch.float32):
        big = dev(g.standard_normal((9, 1100)).astype(np.float32)).to(dtype)
        for first in (0, 1, 3, 8):  # rows that start off 16-byte boundaries
            score_check(P, big[::2, first: first + 997], g.integers(0, 997, (5, 2)).astype(np.int32), 10)
    assert P.token_logprobs(big[:0], top=3)[3].shape == (0, 3)


# -- refusals ---------------------------------------------------------------------------------


def test_refusals(P):
    err = P.AF1Error
    cache = P.KVCache.empty(4, 16, 2, 64, "int8")
    q = torch.zeros((2, 3, 4, 64), dtype=torch.float16, device="cuda")
    table = torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    lens = torch.zeros(2, dtype=torch.int32, device="cuda")

    def code(f, *a, **kw):
        with pytest.raises(err) as e:
            f(*a, **kw)
        return e.value.code

    for kw in (dict(page_size=8), dict(page_size=48), dict(head_dim=96), dict(page_size=512)):
        assert code(P.KVCache.empty, **{**dict(pages=2, page_size=16, kv_heads=1, head_dim=64), **kw}) == -1
    k = torch.zeros((2, 1, 16, 64), dtype=torch.float16)
    assert code(P.KVCache, k, k) == -2  # host memory
    kd = torch.zeros(2 * 16 * 64 + 4, dtype=torch.float16, device="cuda")[4:].view(2, 1, 16, 64)
    assert code(P.KVCache, kd, kd) == -3  # 8-byte aligned
    with pytest.raises(ValueError):
        P.KVCache(kd, kd, lens.float(), lens.float())
    # attention
    assert code(cache.tree_attention, q[:, :, :3], table, lens) == -1  # 3 heads over 2
    assert code(cache.tree_attention, torch.zeros((2, 65, 4, 64), dtype=torch.float16, device="cuda"), table, lens) == -1
    assert code(cache.tree_attention, q, table, lens, workspace=torch.zeros(64, dtype=torch.uint8, device="cuda")) == -8
    assert code(cache.tree_attention, q, table, lens, scale=float("inf")) == -1
    assert code(cache.tree_attention, q, table.cpu(), lens) == -2
    off = torch.zeros(q.numel() + 1, dtype=torch.float16, device="cuda")[1:].view(q.shape)
    assert code(cache.tree_attention, off, table, lens) == -3
    odd = torch.zeros((2, 3, 4, 68), dtype=torch.float16, device="cuda")[..., :64]
    assert code(cache.tree_attention, odd, table, lens) == -3
    for bad in (dict(q=q.float()), dict(pages=table[:1]), dict(lens=lens.long()), dict(mask=table[None]),
                dict(counts=lens[:1]), dict(lse=q.float()), dict(out=q[:1])):
        with pytest.raises(ValueError):
            cache.tree_attention(**{**dict(q=q, pages=table, lens=lens), **bad})
    # append
    kv = torch.zeros((2, 2, 64), dtype=torch.float16, device="cuda")
    idx = torch.zeros(2, dtype=torch.int32, device="cuda")
    rope = torch.zeros((4, 48, 2), dtype=torch.float32, device="cuda")
    assert code(cache.append, kv, kv, table, idx, idx, rope=rope) == -1  # 96 of 64 entries
    assert code(cache.append, kv, kv, table, idx.cpu(), idx) == -2
    for bad in (dict(k=kv.double(), v=kv.double()), dict(v=kv.float()), dict(seq=idx.long()), dict(q_out=kv),
                dict(k_out=kv.float()), dict(rope=rope.half())):
        with pytest.raises(ValueError):
            cache.append(**{**dict(k=kv, v=kv, pages=table, seq=idx, slot=idx), **bad})
    # rope, read, masks, scores
    assert code(P.rope, kv, idx, rope) == -1
    assert code(P.rope, kv, idx, torch.zeros((0, 32, 2), device="cuda")) == -1
    assert code(P.rope, kv.cpu(), idx, rope[:, :16].contiguous()) == -2
    with pytest.raises(ValueError):
        P.rope(kv, idx[:1], rope)
    assert code(cache.read, table, lens, first=-1, count=4) == -1
    assert code(P.tree_mask, torch.zeros((1, 65), dtype=torch.int32, device="cuda")) == -1
    x = torch.zeros((2, 40), dtype=torch.float16, device="cuda")
    assert code(P.token_logprobs, x, top=33) == -1
    assert code(P.token_logprobs, x[:, :5], top=6) == -1
    for t in (0.0, -1.0, float("nan"), float("inf")):
        assert code(P.token_logprobs, x, temperature=t) == -1
    assert code(P.token_logprobs, x.cpu()) == -2
    with pytest.raises(ValueError):
        P.token_logprobs(x, idx[:, None].long())
    with pytest.raises(ValueError):
        P.token_logprobs(x.to(torch.bfloat16))
