"""One workspace for calls of every kind on one stream: what a call leaves in
it (activations, partial sums) must not be taken for another's counters.

Results do not depend on timing, so a call on the shared workspace gives what
it gives on a cleared one, to the bit."""
import numpy as np
import pytest
import torch

import synth
from tests.af1_cases import signs_layer

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06161_gb300 as P
    return P


def make(P, seed, m, n, r):
    return signs_layer(P, synth.layer_signs(seed, m, n, r, 1))


def shared(P, calls):
    """Every call (a function of a workspace, and its bytes) alone on cleared memory, then all of them on one."""
    want = [f(torch.zeros(size, dtype=torch.uint8, device="cuda")).clone() for f, size in calls]
    ws = torch.zeros(max(size for _, size in calls), dtype=torch.uint8, device="cuda")
    for turn in range(3):
        order = list(range(len(calls)))
        np.random.default_rng(turn).shuffle(order)
        for i in order:
            got = calls[i][0](ws)
            assert torch.equal(got, want[i]), (turn, i, int((got != want[i]).sum()))
    P.workspace_status(ws)


def linear(layer, n, tokens):
    x = torch.randn((tokens, n), generator=torch.Generator("cuda").manual_seed(tokens), device="cuda").half()

    def call(ws):
        y = torch.full((tokens, layer.m), float("nan"), dtype=torch.float32, device="cuda")  # rows not written show
        layer.forward_into(x, y, ws)
        return y
    return call, layer.workspace_bytes(tokens)


def attention(P, kind, nodes, group, lens, dim=128):
    g = torch.Generator("cuda").manual_seed(nodes)
    cache = P.KVCache.empty(64, 64, 2, dim, kind)
    k, v = (torch.randn((4096, 2, dim), generator=g, device="cuda").half() for _ in "kv")
    pages = torch.randperm(64, generator=g, device="cuda").to(torch.int32).view(1, 64)
    slot = torch.arange(4096, dtype=torch.int32, device="cuda")
    cache.append(k, v, pages, torch.zeros_like(slot), slot)
    pages = pages.repeat(len(lens), 1)
    q = torch.randn((len(lens), nodes, 2 * group, dim), generator=g, device="cuda").half()
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def call(ws):
        out = torch.full(q.shape, float("nan"), dtype=torch.float32, device="cuda")
        return cache.tree_attention(q, pages, lens, out=out, workspace=ws)
    return call, cache.workspace_bytes(len(lens), nodes, 2 * group)


def test_linears_of_all_lengths(P):
    a, b = make(P, 31, 512, 1024, 200), make(P, 32, 2048, 512, 333)
    shared(P, [linear(a, 1024, t) for t in (1, 7, 16, 100, 333, 2048)] +
              [linear(b, 512, t) for t in (3, 65, 500, 2048)])
    # A rank so large that its activations lie where shorter calls of a layer whose tiles are shared by CTAs end.
    c, d = make(P, 34, 256, 256, 9000), make(P, 35, 512, 8192, 400)
    shared(P, [linear(c, 256, t) for t in (2048, 1200, 5)] + [linear(d, 8192, t) for t in (40, 100, 120, 300, 2048)])


def test_groups_and_single_layers(P):
    layers = [make(P, 40 + i, m, 4096, 150 + 10 * i) for i, m in enumerate((512, 256, 1024))]
    wide = make(P, 50, 256, 256, 9000)

    def group(tokens):
        x = torch.randn((tokens, 4096), generator=torch.Generator("cuda").manual_seed(tokens), device="cuda").half()

        def call(ws):
            ys = [torch.full((tokens, layer.m), float("nan"), dtype=torch.float32, device="cuda") for layer in layers]
            P.forward_multi(layers, x, ys, ws)
            return torch.cat(ys, 1)
        return call, P.workspace_bytes_multi(layers, tokens)
    shared(P, [group(t) for t in (1, 12, 200, 1000)] + [linear(layers[2], 4096, t) for t in (2, 90, 2048)] +
              [linear(wide, 256, t) for t in (2048, 3)])


def test_linears_and_tree_attention(P):
    layer = make(P, 33, 1024, 8192, 400)
    shared(P, [linear(layer, 8192, t) for t in (1, 16, 150, 2048)] +
              [attention(P, "int8", 1, 4, [4000, 30, 0, 1777]), attention(P, "f16", 3, 4, [4090, 3000]),
               attention(P, "int4", 33, 4, [4000, 30, 0, 1777]), attention(P, "e4m3", 64, 8, [2500, 4000])])


def test_more_counters_than_the_head_holds(P):
    """131400 rows: 8216 tiles at 2000 tokens, whose counters lie behind the scratch, where others have theirs."""
    big, c = make(P, 36, 131400, 8192, 64), make(P, 34, 256, 256, 9000)
    shared(P, [linear(big, 8192, 2000), linear(big, 8192, 2), linear(c, 256, 2048), linear(c, 256, 1200)])
