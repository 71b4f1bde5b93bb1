"""examples/drafted_decode.py: the five operators of drafted tokens together, as a program uses them, against the same decoder in fp64 without a cache."""
import importlib.util
import os

import pytest
import torch

from test_gpu_paged_decode import _plain

pytestmark = pytest.mark.gpu
ROOT = os.path.join(os.path.dirname(__file__), "..")


def _example():
    spec = importlib.util.spec_from_file_location("drafted_decode", os.path.join(ROOT, "examples", "drafted_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _models(m, layers=1):
    make = dict(layers=2, width=128, heads=4, kv_heads=2, size=32, vocabulary=97, longest=128, seed=3)
    target, draft = m.Decoder(**make), m.Decoder(**make)
    draft.layers = draft.layers[:layers]
    g = torch.Generator().manual_seed(4)
    return target, draft, [torch.randint(97, (n,), generator=g).tolist() for n in (1, 33, 40, 17)]


def test_trees():
    m = _example()
    assert m.tree(0, 3) == [-1] and m.tree(3, 1) == [-1, 0, 1, 2] and m.tree(2, 2) == [-1, 0, 0, 1, 2]


# As in the test of the decoder over the cache: 3.5 % of the logits' norm in 16 bits, with int8 codes 7.5 %.  A token that is drawn as the likeliest is that of logits so far off: its
# own is below the largest by twice the error at most.
@pytest.mark.parametrize("kind,within", [("same", 0.035), ("int8", 0.075)])
@pytest.mark.parametrize("depth,branch,layers", [(4, 1, 2), (3, 2, 1), (0, 1, 1), (2, 5, 1)])
def test_the_likeliest_tokens(kind, within, depth, branch, layers):
    m = _example()
    target, draft, prompts = _models(m, layers)
    texts, stood, _ = m.generate(target, draft, prompts, 10, depth, branch, kind, page_size=8, temperature=0.0)
    if layers == 2:                                                           # the draft is the target: nearly all stands (near ties aside)
        assert sum(map(sum, stood)) > 0.8 * len(stood) * len(prompts) * (depth + 1)
    for b, (text, prompt) in enumerate(zip(texts, prompts)):
        assert text[:len(prompt)] == prompt and len(text) == len(prompt) + sum(s[b] for s in stood) >= len(prompt) + 10
        for at in range(len(prompt), len(text)):
            want = _plain(target, text[:at])
            assert want[text[at]] >= want.max() - 2 * within * want.norm(), (b, at)


def test_a_draft_that_is_the_target_stands():
    """Drawn tokens: p = q up to the kernels' roundings, so that nearly every draft of a chain stands."""
    m = _example()
    target, draft, prompts = _models(m, 2)
    texts, stood, _ = m.generate(target, draft, prompts, 12, 3, 1, page_size=8, temperature=1.0, seed=2)
    assert sum(map(sum, stood)) >= 0.9 * len(stood) * len(prompts) * 4
    assert all(0 <= t < 97 for text in texts for t in text)
