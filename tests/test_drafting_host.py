"""Refusals, on a host without a GPU, of what follows the logits of drafted
tokens: probabilities, verification, accepted slots, copied pages and the
table of pages."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_06161_gb300", "libaf1.so")
I32, F32, F16 = torch.int32, torch.float32, torch.float16


@pytest.fixture(scope="module")
def P():
    if not os.path.exists(LIB):
        subprocess.run([sys.executable, os.path.join(ROOT, "paper_2609_06161_gb300", "build.py")], check=True)
    import paper_2609_06161_gb300 as P
    return P


def refused(P, code, call, *args):
    assert call(*args) == code
    assert P.last_error() != ""


# -- probabilities -------------------------------------------------------------------


@pytest.mark.parametrize("change", [
    dict(rows=-1), dict(rows=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 30) + 1, ld=1 << 32, probs_ld=1 << 32), dict(ld=99), dict(ld=(1 << 36) + 1),
    dict(probs_ld=99), dict(probs_ld=(1 << 36) + 1), dict(dtype=2), dict(dtype=-1)])
def test_probs_refusals(P, change):
    from paper_2609_06161_gb300 import drafting as D
    a = dict(logits=4096, rows=2, vocab=100, ld=100, probs=8192, probs_ld=100, all_temperature=1.0, dtype=1)
    a.update(change)
    refused(P, -1, D._token_probs, ctypes.byref(D._ProbsArgs(**a)), None)


def test_probs_of_no_rows(P):
    from paper_2609_06161_gb300 import drafting as D
    assert D._token_probs(ctypes.byref(D._ProbsArgs(rows=0, vocab=10, ld=10, probs_ld=10, dtype=1)), None) == 0
    refused(P, -1, D._token_probs, None, None)
    assert P.token_probs(torch.zeros(0, 10)).shape == (0, 10)


def test_probs_arguments(P):
    x = torch.zeros(3, 10)
    for kw in (dict(temperature=torch.zeros(4)), dict(temperature=torch.zeros(3, dtype=F16)),
               dict(top_k=torch.zeros(3)), dict(top_k=torch.zeros(6, dtype=I32)[::2]), dict(min_p=torch.zeros(3, 1)),
               dict(top_k=1.5), dict(top_k=1 << 31), dict(out=torch.zeros(3, 11)), dict(out=torch.zeros(3, 10, dtype=F16)),
               dict(out=torch.zeros(3, 20)[:, ::2])):
        with pytest.raises(ValueError):
            P.token_probs(x, **kw)
    with pytest.raises(ValueError):
        P.token_probs(torch.zeros(3, 10, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        P.token_probs(torch.zeros(10))
    with pytest.raises((P.AF1Error, RuntimeError)):
        P.token_probs(x)  # not on a GPU


def test_probs_overlap(P):
    """Rows of probabilities on rows of logits are refused, unless they are the same ones; between them they are not."""
    from paper_2609_06161_gb300 import drafting as D
    at = 1 << 20  # rows of 100 entries

    def call(**change):
        a = dict(logits=at, rows=3, vocab=100, ld=100, probs=at, probs_ld=100, all_temperature=1.0, dtype=1) | change
        return D._token_probs(ctypes.byref(D._ProbsArgs(**a)), None)

    for change in (dict(dtype=0), dict(probs=at + 4), dict(probs=at - 4), dict(probs_ld=101), dict(probs=at + 1196),
                   dict(probs=at - 1196), dict(ld=200, probs=at + 396, probs_ld=200), dict(ld=1000, probs_ld=500),
                   dict(ld=1000, probs=at + 4396 - 500 * 4, probs_ld=500), dict(ld=1 << 36, probs=at + (2 << 38), rows=1 << 24),
                   dict(dtype=0, probs=at + 196), dict(dtype=0, rows=1), dict(rows=1, ld=200, probs=at + 396)):
        refused(P, -1, lambda: call(**change))
        assert "overlap" in P.last_error(), change
    for change in (dict(), dict(ld=200, probs_ld=200), dict(rows=1, ld=200), dict(probs=at + 1200), dict(probs=at - 1200),
                   dict(ld=200, probs=at + 400, probs_ld=200), dict(ld=200, probs=at - 400, probs_ld=200),
                   dict(ld=1000, probs=at + 400, probs_ld=500), dict(dtype=0, probs=at + 600),
                   dict(dtype=0, ld=400, probs=at + 200, probs_ld=200), dict(rows=1, ld=200, probs=at + 400)):
        call(**change)
        assert "overlap" not in P.last_error(), change


# -- verification --------------------------------------------------------------------


@pytest.mark.parametrize("change", [
    dict(sequences=-1), dict(sequences=65537), dict(nodes=0), dict(nodes=65), dict(vocab=0), dict(vocab=(1 << 22) + 1),
    dict(probs_seq=-1), dict(probs_node=-1), dict(probs_seq=1 << 60), dict(draft=4096, draft_node=-4),
    dict(draft=4096, draft_seq=1 << 61), dict(flags=2), dict(flags=1), dict(reserved=1)])
def test_verify_refusals(P, change):
    from paper_2609_06161_gb300 import drafting as D
    a = dict(probs=4096, probs_seq=300, probs_node=100, tokens=4096, parents=4096, uniforms=4096, path=4096, lengths=4096,
             following=4096, sequences=2, nodes=3, vocab=100)
    a.update(change)
    refused(P, -1, D._verify_tree, ctypes.byref(D._VerifyArgs(**a)), None)


def test_verify_arguments(P):
    from paper_2609_06161_gb300 import drafting as D
    refused(P, -1, D._verify_tree, None, None)
    assert D._verify_tree(ctypes.byref(D._VerifyArgs(sequences=0, nodes=3, vocab=9)), None) == 0
    b, n, v = 2, 3, 10
    good = dict(probs=torch.zeros(b, n, v), tokens=torch.zeros(b, n, dtype=I32), parents=torch.zeros(b, n, dtype=I32),
                uniforms=torch.zeros(b, n))
    for kw in (dict(probs=torch.zeros(b, n, v, dtype=F16)), dict(probs=torch.zeros(b, v)),
               dict(tokens=torch.zeros(b, n, dtype=torch.int64)), dict(parents=torch.zeros(b, n + 1, dtype=I32)),
               dict(uniforms=torch.zeros(b, n, dtype=torch.float64)), dict(uniforms=torch.zeros(b, 2 * n)[:, ::2]),
               dict(draft=torch.zeros(b, n, v + 1)), dict(draft=torch.zeros(b, n, v, dtype=F16)),
               dict(draft=torch.zeros(b, n, 2 * v)[..., ::2]), dict(counts=torch.zeros(3, dtype=I32)), dict(distinct=True),
               dict(out=(torch.zeros(b, n, dtype=I32), torch.zeros(b, dtype=I32), torch.zeros(b))),
               dict(out=(torch.zeros(b, n + 1, dtype=I32), torch.zeros(b, dtype=I32), torch.zeros(b, dtype=I32)))):
        with pytest.raises(ValueError):
            P.verify_tree(**{**good, **kw})
    with pytest.raises((P.AF1Error, RuntimeError)):
        P.verify_tree(**good)  # not on a GPU
    none = P.verify_tree(torch.zeros(0, n, v), torch.zeros(0, n, dtype=I32), torch.zeros(0, n, dtype=I32), torch.zeros(0, n))
    assert [tuple(x.shape) for x in none] == [(0, n), (0,), (0,)]


# -- accepted slots and copied pages -------------------------------------------------


def test_caches_refusals(P):
    from paper_2609_06161_gb300 import drafting as D
    none = (ctypes.c_void_p * 300)()
    refused(P, -1, D._kv_compact, None, 1, 4096, 1, 4, 4, 4096, 4096, 4, 4096, None)
    for n in (0, -1, 257):
        refused(P, -1, D._kv_compact, none, n, 4096, 1, 4, 4, 4096, 4096, 4, 4096, None)
        refused(P, -1, D._kv_copy, none, n, 4096, 1, None)
    for nodes in (0, 65):
        refused(P, -1, D._kv_compact, none, 1, 4096, 1, 4, 4, 4096, 4096, nodes, 4096, None)
    for sequences in (-1, 65537):
        refused(P, -1, D._kv_compact, none, 1, 4096, sequences, 4, 4, 4096, 4096, 4, 4096, None)
    for entries in (-1, (1 << 20) + 1):
        refused(P, -1, D._kv_copy, none, 1, 4096, entries, None)


def test_caches_arguments(P):
    pages, first = torch.zeros(2, 4, dtype=I32), torch.zeros(2, dtype=I32)
    for kw in (dict(first=first.long()), dict(first=torch.zeros(3, dtype=I32)), dict(index=torch.zeros(2, dtype=I32)),
               dict(index=torch.zeros(3, 5, dtype=I32)), dict(counts=torch.zeros(2, 1, dtype=I32)),
               dict(pages=pages.float())):
        with pytest.raises(ValueError):
            P.kv_compact([], **{**dict(pages=pages, first=first, index=torch.zeros(2, 5, dtype=I32), counts=first), **kw})
    for copies in (torch.zeros(4, 2, dtype=I32), torch.zeros(4, 3), torch.zeros(12, dtype=I32), torch.zeros(3, 4, dtype=I32).T):
        with pytest.raises(ValueError):
            P.kv_copy([], copies)
    with pytest.raises((P.AF1Error, RuntimeError)):
        P.kv_copy([], torch.zeros(4, 3, dtype=I32))


# -- the table -----------------------------------------------------------------------


@pytest.mark.parametrize("change", [
    dict(sequences=-1), dict(sequences=1025), dict(columns=0), dict(columns=(1 << 20) + 1), dict(ld=7),
    dict(ld=(1 << 36) + 1), dict(pages=0), dict(pages=1 << 31), dict(page_size=0), dict(page_size=8), dict(page_size=48),
    dict(page_size=512), dict(reserved=1)])
def test_table_refusals(P, change):
    from paper_2609_06161_gb300 import drafting as D
    t = dict(table=4096, refs=4096, sequences=2, columns=8, ld=8, pages=10, page_size=16)
    t.update(change)
    t = ctypes.byref(D._TableDesc(**t))
    refused(P, -1, D._pages_fork, t, 4096, None)
    refused(P, -1, D._pages_release, t, 4096, None)
    refused(P, -1, D._pages_reserve, t, 4096, 4096, 4096, 4096, 4096, 1 << 20, None)
    refused(P, -1, D._pages_workspace, t)


def test_table_workspace(P):
    from paper_2609_06161_gb300 import drafting as D
    t = ctypes.byref(D._TableDesc(table=4096, refs=4096, sequences=3, columns=100, ld=100, pages=10, page_size=16))
    size = D._pages_workspace(t)
    assert size == 3 * 100 * 8
    for pointer, given in ((0, size), (4096 + 128, size), (4096, size - 1)):
        refused(P, -8, D._pages_reserve, t, 4096, 4096, 4096, 4096, pointer, given, None)


def test_table_arguments(P):
    table, refs = torch.full((2, 4), -1, dtype=I32), torch.zeros(9, dtype=I32)
    for args in ((table.long(), refs, 16), (table[0], refs, 16), (table, refs.float(), 16), (table, refs[None], 16)):
        with pytest.raises(ValueError):
            P.PageTable(*args)
    with pytest.raises(P.AF1Error):
        P.PageTable(table, refs, 17)
    t = P.PageTable(table, refs, 16)
    two = torch.zeros(2, dtype=I32)
    for call in (lambda: t.fork(two.long()), lambda: t.fork(torch.zeros(3, dtype=I32)), lambda: t.release(two[None]),
                 lambda: t.reserve(two, two.float()), lambda: t.reserve(two, two, copies=torch.zeros(2, 2, dtype=I32)),
                 lambda: t.reserve(two, two, lacking=torch.zeros(2, dtype=I32))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises((P.AF1Error, RuntimeError)):
        t.fork(two)  # not on a GPU
