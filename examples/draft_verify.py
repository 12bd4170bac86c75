"""Drafted tokens verified in one pass: a small decoder of AF1 layers with a
paged, quantised cache.

    python examples/draft_verify.py [--kind int8] [--tokens 48] [--temperature 0.8]

A decoder with random weights generates greedily. Each step drafts a tree of
tokens (here: the true continuation, found by a plain decoder for the
demonstration, beside wrong guesses), runs the whole tree through the layers
at once, scores every node, and accepts the longest path that greedy decoding
would have taken. The accepted keys and values are written again to the slots
behind the prefix, where the next step expects them.

With a temperature it samples: the tree is verified against the target's
probabilities with random numbers, the accepted slots move behind the prefix
as they are, and the cache's pages are reserved and released step by step.
Nothing but the tokens, and how many they are, comes back to the host.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_06161_gb300 as af1  # noqa: E402


class Decoder:
    """`layers` blocks of attention and SwiGLU around AF1 linears."""

    def __init__(self, layers=2, width=512, heads=8, kv_heads=2, ffn=1024, vocab=1000, kind="int8", slots=512, page=32,
                 seed=0):
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.vocab = heads, kv_heads, width // heads, vocab
        kv = kv_heads * self.dim
        self.embed = torch.randn((vocab, width), generator=self.g, device="cuda").half()
        self.blocks = [dict(q=self.linear(width, width), k=self.linear(kv, width), v=self.linear(kv, width),
                            o=self.linear(width, width), gate=self.linear(ffn, width), up=self.linear(ffn, width),
                            down=self.linear(width, ffn)) for _ in range(layers)]
        self.head = self.linear(vocab, width)
        self.rope = af1.rope_table(slots, self.dim, base=500000.0)
        columns = slots // page
        self.caches = [af1.KVCache.empty(columns, page, kv_heads, self.dim, kind) for _ in range(layers)]
        self.pages = torch.randperm(columns, generator=self.g, device="cuda").to(torch.int32)[None]
        self.workspace = None

    def linear(self, m, n):
        r = af1.rank_for_budget(m, n)
        sign = lambda rows: (torch.randint(0, 2, (rows, r), generator=self.g, device="cuda") * 2 - 1).to(torch.int8)  # noqa: E731
        ones = lambda k, v: torch.full((k,), v, dtype=torch.float16, device="cuda")  # noqa: E731
        return af1.Layer.from_signs(sign(m), sign(n), ones(m, 1.0), ones(r, r ** -0.5), ones(n, n ** -0.5))

    @staticmethod
    def norm(x):
        return (x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).half()

    def write(self, i, k, v, first, positions, q=None):
        """Tokens to the slots from `first` on; the rotated queries."""
        n = k.shape[0]
        seq = torch.zeros(n, dtype=torch.int32, device="cuda")
        slot = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
        return self.caches[i].append(k, v, self.pages, seq, slot, rope=self.rope, positions=positions, q=q)

    def forward(self, tokens, length, depth, mask=None):
        """Logits (float32) of nodes behind `length` cached tokens, and their keys and values of every block. depth:
        position of each node behind the prefix; mask: the tree's, or None for a chain."""
        n = tokens.shape[0]
        x = self.embed[tokens]
        positions = (length + depth).to(torch.int32)
        lens = torch.tensor([length], dtype=torch.int32, device="cuda")
        kept = []
        for i, b in enumerate(self.blocks):
            h = self.norm(x)
            k = b["k"].forward(h).reshape(n, self.kv_heads, self.dim)
            v = b["v"].forward(h).reshape(n, self.kv_heads, self.dim)
            q = self.write(i, k, v, length, positions, b["q"].forward(h).reshape(n, self.heads, self.dim))
            kept.append((k, v))
            if self.workspace is None or self.workspace.numel() < self.caches[i].workspace_bytes(1, n, self.heads):
                self.workspace = self.caches[i].make_workspace(q[None])
            a = self.caches[i].tree_attention(q[None], self.pages, lens, mask=mask, workspace=self.workspace)
            x = x + b["o"].forward(a.reshape(n, -1))
            h = self.norm(x)
            x = x + b["down"].forward_swiglu(b["gate"].forward(h), b["up"].forward(h))
        return self.head.forward(self.norm(x), out_dtype=torch.float32), kept

    def accept(self, kept, nodes, length, depth):
        """The accepted path's keys and values, to the slots behind the prefix."""
        positions = (length + depth[nodes]).to(torch.int32)
        for i, (k, v) in enumerate(kept):
            self.write(i, k[nodes], v[nodes], length, positions)


def greedy(decoder, token, length, steps):
    """Plain decoding, one token a pass, from the last token on."""
    out = []
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    for _ in range(steps):
        logits, _ = decoder.forward(torch.tensor([token], device="cuda"), length, zero)
        token = int(af1.token_logprobs(logits, top=1)[3][0, 0])
        out.append(token)
        length += 1
    return out


def draft(truth, vocab, g):
    """A tree whose root is the last token: three guesses at every depth, one of them the true one (until the draft
    errs), each under the true one before. Returns (tokens, parents)."""
    tokens, parents, parent = [truth[0]], [-1], 0
    errs = 1 + int(torch.randint(1, len(truth), (1,), generator=g))
    for d, t in enumerate(truth[1:], 1):
        guesses = torch.randint(0, vocab, (3,), generator=g).tolist()
        at = int(torch.randint(0, 3, (1,), generator=g))
        if d < errs:
            guesses[at] = t
        first = len(tokens)
        tokens += guesses
        parents += [parent] * 3
        parent = first + at
    return tokens, parents


def run(kind="int8", steps=48, drafted=5, prompt=9, seed=0, say=print):
    """(tokens by plain decoding, tokens by drafts, passes of the drafts, largest difference of a log-probability)."""
    decoder = Decoder(kind=kind, seed=seed)
    g = torch.Generator().manual_seed(seed)
    start = torch.randint(0, decoder.vocab, (prompt,), generator=g).cuda()
    logits, _ = decoder.forward(start, 0, torch.arange(prompt, device="cuda"))
    first = int(logits[-1].argmax())
    plain = [first] + greedy(decoder, first, prompt, steps + drafted)

    decoder.forward(start, 0, torch.arange(prompt, device="cuda"))  # the cache as after the prompt
    found, length, passes, off = [first], prompt, 0, 0.0
    while len(found) <= steps:
        at = len(found) - 1
        tokens, parents = draft(plain[at: at + drafted], decoder.vocab, g)
        parents = torch.tensor(parents, dtype=torch.int32, device="cuda")
        depth = torch.zeros(len(tokens), dtype=torch.int64, device="cuda")
        for i in range(1, len(tokens)):
            depth[i] = depth[parents[i]] + 1
        logits, kept = decoder.forward(torch.tensor(tokens, device="cuda"), length, depth,
                                       mask=af1.tree_mask(parents[None]))
        passes += 1
        # The greedy token of every node, and the scores of the children under it.
        children = torch.full((len(tokens), 3), -1, dtype=torch.int32, device="cuda")
        nodes_of = {}
        for i in range(1, len(tokens)):
            nodes_of.setdefault(int(parents[i]), []).append(i)
        for p, c in nodes_of.items():
            children[p, : len(c)] = torch.tensor([tokens[i] for i in c], dtype=torch.int32, device="cuda")
        logprobs, _, _, best = af1.token_logprobs(logits, children, top=1)
        path = [0]
        while True:
            node, want = path[-1], int(best[path[-1], 0])
            found.append(want)
            hit = [i for i in nodes_of.get(node, []) if tokens[i] == want]
            if not hit:
                break
            path.append(hit[0])
        chosen = torch.log_softmax(logits, -1)
        for p, c in nodes_of.items():
            off = max(off, float((logprobs[p, : len(c)] - chosen[p, [tokens[i] for i in c]]).abs().max()))
        decoder.accept(kept, torch.tensor(path, device="cuda"), length, depth)
        length += len(path)
    torch.cuda.synchronize()
    af1.workspace_status(decoder.workspace)
    say(f"{kind}: {steps} tokens in {passes} passes of drafts ({steps / passes:.2f} a pass); "
        f"{sum(a == b for a, b in zip(plain, found[: steps]))} of {steps} as by plain decoding")
    return plain[:steps], found[:steps], passes, off


def sample(kind="int8", steps=48, drafted=5, prompt=9, seed=0, temperature=0.8, top_k=50, say=print):
    """(tokens by plain greedy decoding, sampled tokens, passes): guesses around the greedy text, verified at this
    temperature (0: what comes out is the greedy text)."""
    decoder = Decoder(kind=kind, seed=seed)
    g = torch.Generator().manual_seed(seed)
    start = torch.randint(0, decoder.vocab, (prompt,), generator=g).cuda()
    logits, _ = decoder.forward(start, 0, torch.arange(prompt, device="cuda"))
    first = int(logits[-1].argmax())
    plain = [first] + greedy(decoder, first, prompt, steps + drafted)

    # The same cache, now through a table of pages that grows with the text.
    one = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")  # noqa: E731
    cache = decoder.caches[0]
    table = af1.PageTable.empty(1, decoder.pages.shape[1], cache.pages, cache.page_size)
    decoder.pages = table.table
    lens = one(0)
    table.reserve(lens, one(prompt))
    decoder.forward(start, 0, torch.arange(prompt, device="cuda"))
    lens += prompt
    found, length, passes = [first], prompt, 0
    while len(found) <= steps:
        at = len(found) - 1
        tokens, parents = draft([found[-1]] + plain[at + 1: at + drafted], decoder.vocab, g)
        n = len(tokens)
        depth = torch.zeros(n, dtype=torch.int64)
        for i in range(1, n):
            depth[i] = depth[parents[i]] + 1
        tokens = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        parents = torch.tensor(parents, dtype=torch.int32, device="cuda")[None]
        copies, lacking = table.reserve(lens, one(n))
        af1.kv_copy(decoder.caches, copies)  # of pages that other sequences hold, too: there are none here
        logits, _ = decoder.forward(tokens.long(), length, depth.cuda(), mask=af1.tree_mask(parents))
        probs = af1.token_probs(logits, temperature=temperature, top_k=top_k)
        path, lengths, following = af1.verify_tree(probs[None], tokens[None], parents, torch.rand((1, n), generator=g).cuda())
        af1.kv_compact(decoder.caches, table.table, lens, path, lengths)
        lens += lengths
        table.release(lens)
        passes += 1
        accepted = path[0, 1: int(lengths[0])].long()
        found += tokens[accepted].tolist() + [int(following[0])]
        length += int(lengths[0])
        assert int(lacking[0]) == 0, "no pages are left"
    say(f"{kind} at temperature {temperature}: {len(found) - 1} tokens in {passes} passes of drafts "
        f"({(len(found) - 1) / passes:.2f} a pass)")
    return plain[:steps], found[:steps], passes


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--kind", choices=["f16", "int8", "e4m3", "int4"], default="int8")
    p.add_argument("--tokens", type=int, default=48)
    p.add_argument("--temperature", type=float, default=None, help="sample at this temperature")
    a = p.parse_args()
    if a.temperature is None:
        run(a.kind, a.tokens)
    else:
        sample(a.kind, a.tokens, temperature=a.temperature)
