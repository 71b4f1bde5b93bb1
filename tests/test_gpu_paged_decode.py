"""examples/paged_decode.py: chunks of prompts and single tokens over the paged cache against the same decoder in fp64 without a cache."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


def _example():
    spec = importlib.util.spec_from_file_location("paged_decode", os.path.join(os.path.dirname(__file__), "..", "examples", "paged_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _plain(model, text):
    """Logits behind the text's last token, fp64 on the CPU, every token anew."""
    def d(t): return t.cpu().double()
    def norm(t): return t / (t * t).mean(1, keepdim=True).add(1e-6).sqrt()
    n, H, K, D = len(text), model.heads, model.kv_heads, model.size
    x = d(model.tokens)[text] + d(model.positions)[:n]
    hidden = torch.ones(n, n, dtype=torch.bool).triu(1)
    for w in model.layers:
        q, k, v = (norm(x) @ d(w["qkv"])).split([H * D, K * D, K * D], 1)
        q, k, v = q.view(n, H, D).transpose(0, 1), k.view(n, K, D).transpose(0, 1), v.view(n, K, D).transpose(0, 1)
        k, v = k.repeat_interleave(H // K, 0), v.repeat_interleave(H // K, 0)
        p = (q @ k.transpose(1, 2) / D ** 0.5).masked_fill(hidden, float("-inf")).softmax(2)
        x = x + (p @ v).transpose(0, 1).reshape(n, H * D) @ d(w["out"])
        x = x + torch.nn.functional.silu(norm(x) @ d(w["up"])) @ d(w["down"])
    return (norm(x[-1:]) @ d(model.read_out))[0]


# Two layers of 9 roundings each to 2^-11 of the value at most, with 4 for what later layers make of them: 18 * 4 * 2^-11 = 3.5 %.  Codes are off by half a step
# at most: int8 0.5 / 127 of the largest of 32 elements (2.5 times their root mean square or so) is 1 %, e4m3 2^-4 = 6.3 %, for K and V of two layers, the
# softmax and the layers between damping as often as not: 4 times that.
@pytest.mark.parametrize("kind,within", [("same", 0.035), ("int8", 0.075), ("e4m3", 0.285)])
@pytest.mark.parametrize("chunk", [5, 64])
def test_generates_what_the_decoder_without_a_cache_would(kind, within, chunk):
    m = _example()
    model = m.Decoder(layers=2, width=128, heads=4, kv_heads=2, size=32, vocabulary=97, longest=128, seed=3)
    g = torch.Generator().manual_seed(4)
    prompts = [torch.randint(97, (n,), generator=g).tolist() for n in (1, 33, 64, 17)]
    texts, logits, _ = m.generate(model, prompts, 6, chunk, kind, page_size=8)
    for text, prompt, got in zip(texts, prompts, logits.cpu().double()):
        assert text[:len(prompt)] == prompt and len(text) == len(prompt) + 6
        want = _plain(model, text)
        assert (got - want).norm() <= within * want.norm(), ((got - want).norm() / want.norm()).item()


def test_parked_sequences_continue_alike():
    """A 16-bit cache read into host memory and written to other pages holds the same bits: the same texts and logits come of it."""
    m = _example()
    model = m.Decoder(layers=2, width=128, heads=4, kv_heads=2, size=32, vocabulary=97, longest=128, seed=3)
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(97, (n,), generator=g).tolist() for n in (40, 1, 19)]
    stay, moved = (m.generate(model, prompts, 4, 16, "same", page_size=8, park=p) for p in (0, 2))
    assert stay[0] == moved[0] and torch.equal(stay[1], moved[1])
