"""Text generation for several sequences at once over a paged key / value cache: prompts in chunks, sequences parked in host memory to make
room and brought back to other pages, then a token of every sequence at a time.

A small decoder with random weights (synthetic: there is no checkpoint) whose products, norms, sums, cache and attention are this library's; torch holds
the tensors, looks up embeddings and picks the next token.  Run on a GPU:

    python examples/paged_decode.py [--cache same|e4m3|int8] [--sequences 8] [--prompt 700] [--chunk 256] [--new 64]
                                    [--park 1] [--seed 0]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2507_11978_amd as nt  # noqa: E402

CACHE_TYPES = {"same": None, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}


class Pages:
    """Which pages of the cache each sequence has: one list for all layers, handed out as the sequences grow."""

    def __init__(self, sequences, pages, page_size):
        self.size, self.free = page_size, list(range(pages))[::-1]
        self.of = [[] for _ in range(sequences)]
        self.length = [0] * sequences

    def grow(self, counts):
        """Room for counts[b] more tokens of sequence b: their slots and positions, and the arguments of the attention over them (on the host)."""
        slots, positions, starts = [], [], [0]
        for b, n in enumerate(counts):
            for p in range(self.length[b], self.length[b] + n):
                if p // self.size == len(self.of[b]):
                    self.of[b].append(self.free.pop())
                slots.append(self.of[b][p // self.size] * self.size + p % self.size)
                positions.append(p)
            self.length[b] += n
            starts.append(len(slots))
        width = max(len(p) for p in self.of)
        table = [p + [-1] * (width - len(p)) for p in self.of]             # (-1 names no page; nothing reads it)
        return slots, positions, table, starts, list(self.length)

    def slots(self, b):
        return [self.of[b][p // self.size] * self.size + p % self.size for p in range(self.length[b])]

    def give_back(self, b):
        self.free = self.of[b][::-1] + self.free
        self.of[b] = []

    def take_again(self, b):
        self.of[b] = [self.free.pop() for _ in range(-(-self.length[b] // self.size))]


class Decoder:
    def __init__(self, layers=4, width=1024, heads=16, kv_heads=4, size=64, vocabulary=4096, longest=4096, dtype=torch.float16, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, generator=g) * shape[0] ** -0.5).to(dtype).to(device)

        self.heads, self.kv_heads, self.size, self.width, self.dtype, self.device = heads, kv_heads, size, width, dtype, device
        self.tokens = (torch.randn(vocabulary, width, generator=g)).to(dtype).to(device)
        self.positions = (torch.randn(longest, width, generator=g)).to(dtype).to(device)
        self.layers = [dict(qkv=weight(width, (heads + 2 * kv_heads) * size), out=weight(heads * size, width), up=weight(width, 4 * width),
                            down=weight(4 * width, width)) for _ in range(layers)]
        self.read_out = weight(width, vocabulary)

    def make_cache(self, pages, page_size, kind):
        """A layer's K and V, and their scales where the cache is narrower than the tokens."""
        shape = (pages, page_size, self.kv_heads, self.size)
        of = CACHE_TYPES[kind] or self.dtype
        self.cache = [[torch.empty(shape, dtype=of, device=self.device) for _ in range(2)] +
                      [None if kind == "same" else torch.empty(shape[:3], dtype=torch.float32, device=self.device) for _ in range(2)] for _ in self.layers]

    def read(self, slots):
        """K and V of these slots in all layers, in the tokens' type, in host memory."""
        slots = torch.tensor(slots, dtype=torch.int64, device=self.device)
        shape = (len(slots), self.kv_heads, self.size)
        return [[t.cpu() for t in nt.cache_read(c[0], c[1], slots, self._new(*shape), self._new(*shape), c[2], c[3])] for c in self.cache]

    def write(self, slots, held):
        slots = torch.tensor(slots, dtype=torch.int64, device=self.device)
        for c, (k, v) in zip(self.cache, held):
            nt.cache_write(k.to(self.device), v.to(self.device), slots, *c)

    def _new(self, *shape):
        return torch.empty(*shape, dtype=self.dtype, device=self.device)

    def __call__(self, ids, slots, positions, table, starts, lengths):
        """Logits [sequences, vocabulary] behind each sequence's last new token; the new tokens' K and V are in the cache afterwards."""
        def to(x, t): return torch.tensor(x, dtype=t, device=self.device)
        longest, most = max(lengths), max(b - a for a, b in zip(starts, starts[1:]))
        last = to([s - 1 for s in starts[1:]], torch.int64)
        slots, positions, table, starts, lengths = (to(slots, torch.int64), to(positions, torch.int64), to(table, torch.int32), to(starts, torch.int32),
                                                    to(lengths, torch.int32))
        T, q_width, kv_width = len(slots), self.heads * self.size, self.kv_heads * self.size
        x = nt.add(self.tokens[ids].flatten(), self.positions[positions].flatten(), self._new(T * self.width)).view(T, self.width)
        for w, cache in zip(self.layers, self.cache):
            qkv = nt.gemm(nt.rms_norm(x, self._new(T, self.width)), w["qkv"], self._new(T, q_width + 2 * kv_width))
            q = qkv[:, :q_width].unflatten(1, (self.heads, self.size))
            k, v = (t.unflatten(1, (self.kv_heads, self.size)) for t in qkv[:, q_width:].split(kv_width, 1))
            nt.cache_write(k, v, slots, *cache)
            seen = self._new(T, self.heads, self.size)
            nt.sdpa_paged(q, cache[0], cache[1], table, starts, lengths, seen, cache[2], cache[3], max_queries=most, max_length=longest)
            x = nt.addmm(x, seen.flatten(1), w["out"], self._new(T, self.width))
            up = nt.addmm(None, nt.rms_norm(x, self._new(T, self.width)), w["up"], self._new(T, 4 * self.width), beta=0.0, act="silu")
            x = nt.addmm(x, up, w["down"], self._new(T, self.width))
        x = x[last]
        return nt.gemm(nt.rms_norm(x, self._new(*x.shape)), self.read_out, self._new(len(last), self.read_out.shape[1]))


def generate(model, prompts, new, chunk, kind="same", page_size=16, park=0):
    """`new` tokens behind each prompt, the likeliest each time, the first `park` sequences parked between prompt and steps; returns the texts, the last
    logits and the seconds of (prompts, parking, steps)."""
    texts = [list(p) for p in prompts]
    most = max(len(t) for t in texts) + new
    if not all(texts) or most > len(model.positions):
        raise ValueError(f"prompts have 1 to {len(model.positions) - new} tokens here")
    pages = Pages(len(texts), len(texts) * -(-most // page_size), page_size)
    model.make_cache(len(pages.free), page_size, kind)
    longest = max(len(t) for t in texts)
    logits = torch.empty(len(texts), model.read_out.shape[1], dtype=model.dtype, device=model.device)
    torch.cuda.synchronize()
    began = time.perf_counter()
    for at in range(0, longest, chunk):
        counts = [min(chunk, max(0, len(t) - at)) for t in texts]          # (a shorter prompt has no tokens in the last chunks)
        ids = torch.tensor([i for t, n in zip(texts, counts) for i in t[at:at + n]], device=model.device)
        got = model(ids, *pages.grow(counts))
        for b, n in enumerate(counts):
            if n:
                logits[b] = got[b]
    torch.cuda.synchronize()
    filled = time.perf_counter()
    parked = range(min(park, len(texts)))
    held = [model.read(pages.slots(b)) for b in parked]
    for b in parked:
        pages.give_back(b)
    for b in parked:
        pages.take_again(b)
        model.write(pages.slots(b), held[b])
    torch.cuda.synchronize()
    back = time.perf_counter()
    for _ in range(new):
        ids = logits.argmax(1)
        for t, i in zip(texts, ids.tolist()):
            t.append(i)
        logits = model(ids, *pages.grow([1] * len(texts)))
    torch.cuda.synchronize()
    return texts, logits, (filled - began, back - filled, time.perf_counter() - back)


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--cache", choices=sorted(CACHE_TYPES), default="int8")
    for name, value in (("sequences", 8), ("prompt", 700), ("chunk", 256), ("new", 64), ("park", 1), ("seed", 0)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    model = Decoder(seed=a.seed)
    g = torch.Generator().manual_seed(a.seed + 1)
    lengths = torch.randint(1, a.prompt + 1, (a.sequences,), generator=g).tolist()
    prompts = [torch.randint(len(model.tokens), (n,), generator=g).tolist() for n in lengths]
    generate(model, prompts, 2, a.chunk, a.cache, park=a.park)       # (first calls load kernels and make the workspace)
    texts, _, (filling, parking, stepping) = generate(model, prompts, a.new, a.chunk, a.cache, park=a.park)
    print(f"{a.sequences} sequences, cache {a.cache}: {sum(lengths)} prompt tokens in {1e3 * filling:.1f} ms, {a.park} parked and back in "
          f"{1e3 * parking:.1f} ms, {a.new} steps of {1e3 * stepping / max(1, a.new):.2f} ms ({a.sequences * a.new / stepping if stepping else 0:.0f} tokens/s)")
    print("first text ends with", texts[0][-min(8, a.new):] if a.new else [])


if __name__ == "__main__":
    main()
