"""CPU test of examples/drafted_decode.py's bookkeeping: sequences that keep more of their drafts than others stay within their pages and positions.  The library's calls are the oracle's
here, the decoders give even odds, and how many drafts stand is given."""
import importlib.util
import os
import types

import pytest
import torch

from oracle import tree as ot

ROOT = os.path.join(os.path.dirname(__file__), "..")


def _example():
    spec = importlib.util.spec_from_file_location("drafted_decode", os.path.join(ROOT, "examples", "drafted_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _library(stands):
    def cache_fit(lengths, counts, page, table, held, free, free_count, starts, new_lengths, slots, positions):
        pages, have, stack = table.numpy(), held.tolist(), free.tolist()
        s, n, at, p, top = ot.fit(lengths.tolist(), counts.tolist(), page, pages, have, stack, free_count.item(), len(slots))
        for t, x in ((held, have), (free, stack), (free_count, [top]), (starts, s), (new_lengths, n), (slots, at), (positions, p)):
            t.copy_(torch.tensor(x))

    def tree_masks(parents, starts, masks, depths, lengths, positions):
        for b, (lo, hi) in enumerate(zip(starts.tolist(), starts.tolist()[1:])):
            depths[lo:hi] = torch.tensor(ot.ancestors(parents[lo:hi].tolist())[1], dtype=torch.int32)
            positions[lo:hi] = lengths[b] - (hi - lo) + depths[lo:hi]

    def verify_tree(target, draft, ids, parents, starts, u, r, path, accepted, following, lengths, after):
        for b, (lo, hi) in enumerate(zip(starts.tolist(), starts.tolist()[1:])):
            chain, p = [0], parents[lo:hi].tolist()
            while len(chain) < min(stands[b], path.shape[1]) and chain[-1] in p:
                chain.append(p.index(chain[-1]))
            path[b] = torch.tensor(chain + [-1] * (path.shape[1] - len(chain)))
            accepted[b], following[b], after[b] = len(chain), b, lengths[b] - (hi - lo) + len(chain)
    return types.SimpleNamespace(cache_fit=cache_fit, tree_masks=tree_masks, verify_tree=verify_tree, cache_compact=lambda *a: None)


class _Decoder:
    def __init__(self, longest):
        self.device, self.positions, self.read_out, self.cache = "cpu", torch.zeros(longest, 1), torch.zeros(1, 11), []

    def make_cache(self, pages, page_size, kind):
        pass


@pytest.mark.parametrize("depth,branch,new,stands", [(4, 2, 64, [5, 1, 2]), (4, 1, 20, [1, 5, 5]), (1, 3, 7, [2, 1, 1]), (0, 1, 9, [1, 1, 1]), (6, 1, 30, [7, 7, 7])])
def test_the_fast_wait_for_the_slow(monkeypatch, depth, branch, new, stands):
    m = _example()
    n, lengths = len(m.tree(depth, branch)), [40, 1, 23]
    longest = max(lengths) + new + 2 * n + 2                                   # what the function asks for
    monkeypatch.setattr(m, "nt", _library(stands))
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)

    def seen(self, ids, slots, positions, starts, masks, most):
        assert (slots >= 0).all(), "tokens without a page"
        assert (positions < longest).all(), "positions beyond the decoder's"
        return torch.zeros((len(ids), 11))
    monkeypatch.setattr(m.Sequences, "__call__", seen)
    prompts = [[3] * k for k in lengths]
    texts, stood, _ = m.generate(_Decoder(longest), _Decoder(longest), prompts, new, depth, branch, page_size=8)
    for b, (text, prompt) in enumerate(zip(texts, prompts)):
        assert text[:len(prompt)] == prompt and len(text) == len(prompt) + sum(s[b] for s in stood) >= len(prompt) + new
    with pytest.raises(ValueError):
        m.generate(_Decoder(longest - 1), _Decoder(longest - 1), prompts, new, depth, branch, page_size=8)
