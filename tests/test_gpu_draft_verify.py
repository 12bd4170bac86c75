"""The example that runs the step around the linears as a program does:
drafted tokens must give what plain decoding gives.

Both see the same keys and values (a cache holds them as a function of the
inputs, whichever pass wrote them) and differ in the order of FP32 sums and in
FP16 roundings of weights; a random decoder's best token stands off the
second by far more than that nearly always, so nearly all tokens agree until
the first difference, after which the texts may part."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f16", "int8", "e4m3", "int4"])
def test_drafts_give_the_plain_text(kind):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import draft_verify
    finally:
        sys.path.pop(0)
    plain, found, passes, off = draft_verify.run(kind, steps=40, say=lambda _: None)
    same = next((i for i, (a, b) in enumerate(zip(plain, found)) if a != b), len(plain))
    assert same >= 20, (plain, found)
    assert passes < 40  # drafts were accepted
    assert off <= 1e-5  # FP32 log-probabilities against torch's


def test_one_pass_over_a_tree_is_every_path_of_it():
    """Logits of a tree's nodes against each path run as a chain."""
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import draft_verify
    finally:
        sys.path.pop(0)
    import paper_2609_06161_gb300 as P
    d = draft_verify.Decoder(kind="int8", seed=3)
    prompt = torch.arange(11, device="cuda") * 7
    d.forward(prompt, 0, torch.arange(11, device="cuda"))
    tokens = torch.tensor([5, 9, 200, 31, 77, 8], device="cuda")
    parents = torch.tensor([-1, 0, 0, 1, 2, 4], dtype=torch.int32, device="cuda")
    depth = torch.tensor([0, 1, 1, 2, 2, 3], device="cuda")
    tree, _ = d.forward(tokens, 11, depth, mask=P.tree_mask(parents[None]))
    for path in ([0, 1, 3], [0, 2, 4, 5]):
        chain, _ = d.forward(tokens[path], 11, torch.arange(len(path), device="cuda"))
        # The same keys and values; FP16 activations (2^-11) through two blocks of layers.
        assert (tree[path] - chain).abs().max() <= 2.0 ** -5 * chain.abs().max()
