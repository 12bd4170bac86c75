"""Host side of the step around the linears: rotary frequencies against their
formulas, and refusals that need no GPU."""
import ctypes
import math
import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_06161_gb300", "libaf1.so")


@pytest.fixture(scope="module")
def P():
    if not os.path.exists(LIB):
        subprocess.run([sys.executable, os.path.join(ROOT, "paper_2609_06161_gb300", "build.py")], check=True)
    import paper_2609_06161_gb300 as P
    return P


@pytest.mark.parametrize("dim", [4, 64, 128, 256])
@pytest.mark.parametrize("scaling", [None, "linear", "base", "bands", "ramp"])
def test_frequencies(P, dim, scaling):
    base, factor, low, high, original = 500000.0, 8.0, 1.0, 4.0, 8192.0
    got, att = P.rope_frequencies(dim, base, scaling, factor, low, high, original)
    i = np.arange(dim // 2)
    f = base ** (-2.0 * i / dim)
    want_att = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "base":
        f = (base * factor ** (dim / (dim - 2.0))) ** (-2.0 * i / dim)
        np.testing.assert_allclose(got[-1], base ** (-2.0 * i[-1] / dim) / factor, rtol=1e-12)  # the slowest, divided
    elif scaling == "bands":
        turns = original * f / (2 * math.pi)  # of a pair within the original context
        g = np.clip((turns - low) / (high - low), 0, 1)
        f = (1 - g) * f / factor + g * f
    elif scaling == "ramp":
        e = lambda beta: dim * math.log(original / (2 * math.pi * beta)) / (2 * math.log(base))  # noqa: E731
        i0, i1 = max(0, math.floor(e(high))), min(dim - 1, math.ceil(e(low)))
        g = np.clip((i - i0) / (i1 - i0), 0, 1)
        f = (1 - g) * f + g * f / factor
        want_att = 0.1 * math.log(factor) + 1
    np.testing.assert_allclose(got, f, rtol=1e-12)
    assert att == pytest.approx(want_att, rel=1e-15)
    assert P.rope_frequencies(dim, base, scaling, factor, low, high, original, attention=0.75)[1] == 0.75


def test_default_bounds(P):
    """Of each scaling its own: what is between the bounds, and what not."""
    kw = dict(base=10000.0, factor=4.0, original=4096.0)
    for scaling, low, high in (("bands", 1.0, 4.0), ("ramp", 1.0, 32.0)):
        default, _ = P.rope_frequencies(128, scaling=scaling, **kw)
        assert default == P.rope_frequencies(128, scaling=scaling, low=low, high=high, **kw)[0]
        turns = 4096.0 * 10000.0 ** (-2.0 * np.arange(64) / 128) / (2 * math.pi)
        kept = np.isclose(default, 10000.0 ** (-2.0 * np.arange(64) / 128), rtol=1e-12)
        assert kept[turns > high * 1.3].all() and not kept[turns < high / 1.3].any()


def test_ramp_without_a_span(P):
    """Both bounds at one index: a step behind it."""
    for original, keeps in ((2 * math.pi * 0.01, 1), (2 * math.pi * 1e9, 32)):  # before the first index, after the last
        got, _ = P.rope_frequencies(64, 10000.0, "ramp", 8.0, 1.0, 2.0, original)
        f = 10000.0 ** (-2.0 * np.arange(32) / 64)
        np.testing.assert_allclose(got, np.where(np.arange(32) < keeps, f, f / 8), rtol=1e-12)


def test_refusals(P):
    for kw in (dict(dim=0), dict(dim=3), dict(dim=258), dict(dim=64, base=1.0), dict(dim=64, base=float("nan")),
               dict(dim=64, scaling="linear", factor=0.5), dict(dim=64, scaling="bands", original=0.0),
               dict(dim=64, scaling="ramp", original=4096.0, low=4.0, high=4.0), dict(dim=64, attention=-1.0),
               dict(dim=2, scaling="base", factor=2.0)):
        with pytest.raises(P.AF1Error) as e:
            P.rope_frequencies(**kw)
        assert e.value.code == -1, kw
    with pytest.raises(ValueError):
        P.rope_frequencies(64, scaling="other")
    lib = P._lib
    assert lib.af1_rope(None, None) == -1
    assert lib.af1_kv_create(None, None) == -1
    h = ctypes.c_void_p()
    assert lib.af1_kv_create(None, ctypes.byref(h)) == -1 and not h.value
    assert lib.af1_kv_append(None, None, None) == -1
    assert lib.af1_tree_attention(None, None, None, 0, None) == -1
    assert lib.af1_tree_workspace_bytes(None, 1, 1, 1) == -1
    assert lib.af1_tree_mask(None, 1, 65, None, None) == -1
    assert lib.af1_token_logprobs(None, None) == -1
    assert "args is NULL" in P.last_error()
    lib.af1_kv_free(None)  # NULL-safe
    from paper_2609_06161_gb300 import attention as A
    d = A._KvDesc(1, 48, 1, 64, 0, None, None, None, None)
    assert lib.af1_kv_create(ctypes.byref(d), ctypes.byref(h)) == -1
    assert "page_size" in P.last_error()
    for rows, vocab, top, temperature in ((1, 0, 0, 1.0), (1, 8, 0, 0.0), (-1, 8, 0, 1.0)):
        a = A._LogprobArgs(None, rows, vocab, vocab, None, 0, None, None, None, None, top, 0, temperature, 0)
        assert lib.af1_token_logprobs(ctypes.byref(a), None) == -1


def test_struct_layouts_match_the_header(P):
    """Field names and order of the ctypes structures are those of include/af1.h."""
    import re
    from paper_2609_06161_gb300 import attention as A
    src = open(os.path.join(ROOT, "include", "af1.h")).read()
    for name, cls in (("af1_rope_params", A._RopeParams), ("af1_rope_args", A._RopeArgs), ("af1_kv_desc", A._KvDesc),
                      ("af1_kv_append_args", A._AppendArgs), ("af1_tree_args", A._TreeArgs),
                      ("af1_logprob_args", A._LogprobArgs)):
        body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct %s \{(.*?)\}" % name, src, re.S).group(1), flags=re.S)
        fields = []
        for decl in body.split(";"):
            decl = decl.strip()
            if not decl:
                continue
            kind, names = re.match(r"((?:const )?\w+)\s*(.*)", decl, re.S).groups()
            for n in names.split(","):
                size = 8 if "*" in n or kind in ("int64_t", "double") else 4
                fields.append((n.strip(" *\n"), size))
        got = [(n, ctypes.sizeof(t)) for n, t in cls._fields_]
        assert got == fields, name
