"""Text generation with drafted tokens over a paged key / value cache: a small draft decoder proposes a tree of tokens behind every sequence's text, the target decoder
looks at the whole tree at once, and what stands by given random numbers is kept.  Pages, slots, positions, masks, verification and the move of what stands are
worked out on the GPU; the host reads back the texts, and whether there is enough of them.

Both decoders are those of paged_decode.py, with random weights (the draft is the target with fewer layers).  Run on a GPU:

    python examples/drafted_decode.py [--sequences 8] [--prompt 300] [--depth 4] [--branch 2] [--new 64] [--cache same|e4m3|int8] [--temperature 1.0] [--seed 0]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paged_decode import Decoder, nt  # noqa: E402


def tree(depth, branch):
    """Parents of a tree: the root, `branch` drafts behind it, each the beginning of a chain."""
    parents = [-1] + [0] * (branch if depth else 0)
    for level in range(1, depth):
        parents += [len(parents) - branch + i for i in range(branch)]
    return parents


class Sequences:
    """A batch's pages and lengths, on the GPU, for one decoder's cache."""

    def __init__(self, model, batch, pages, page_size, width, kind):
        self.model, self.page, self.B, dev = model, page_size, batch, model.device
        model.make_cache(pages, page_size, kind)
        self.table = torch.full((batch, width), -1, dtype=torch.int32, device=dev)
        self.held, self.lengths = (torch.zeros(batch, dtype=torch.int32, device=dev) for _ in range(2))
        self.free, self.free_count = torch.arange(pages, dtype=torch.int32, device=dev), torch.full((1,), pages, dtype=torch.int32, device=dev)

    def grow(self, counts, total):
        """Room for counts[b] more tokens of each sequence, `total` in all: their slots, positions and starts."""
        dev = self.table.device
        starts = torch.empty(self.B + 1, dtype=torch.int32, device=dev)
        slots, positions = torch.empty(total, dtype=torch.int64, device=dev), torch.empty(total, dtype=torch.int32, device=dev)
        nt.cache_fit(self.lengths, counts, self.page, self.table, self.held, self.free, self.free_count, starts, self.lengths, slots, positions)
        return slots, positions, starts

    def __call__(self, ids, slots, positions, starts, masks, most):
        """Logits behind every one of these new tokens; `masks`: of a tree's, None: each sees those before it."""
        m, T = self.model, len(ids)
        q_width, kv_width = m.heads * m.size, m.kv_heads * m.size
        x = nt.add(m.tokens[ids].flatten(), m.positions[positions].flatten(), m._new(T * m.width)).view(T, m.width)
        for w, cache in zip(m.layers, m.cache):
            qkv = nt.gemm(nt.rms_norm(x, m._new(T, m.width)), w["qkv"], m._new(T, q_width + 2 * kv_width))
            q = qkv[:, :q_width].unflatten(1, (m.heads, m.size))
            k, v = (t.unflatten(1, (m.kv_heads, m.size)) for t in qkv[:, q_width:].split(kv_width, 1))
            nt.cache_write(k, v, slots, *cache)
            seen = m._new(T, m.heads, m.size)
            if masks is None:
                nt.sdpa_paged(q, cache[0], cache[1], self.table, starts, self.lengths, seen, cache[2], cache[3], max_queries=most)
            else:
                nt.sdpa_paged_tree(q, cache[0], cache[1], self.table, starts, self.lengths, masks, seen, cache[2], cache[3], max_queries=most)
            x = nt.addmm(x, seen.flatten(1), w["out"], m._new(T, m.width))
            up = nt.addmm(None, nt.rms_norm(x, m._new(T, m.width)), w["up"], m._new(T, 4 * m.width), beta=0.0, act="silu")
            x = nt.addmm(x, up, w["down"], m._new(T, m.width))
        return nt.gemm(nt.rms_norm(x, m._new(*x.shape)), m.read_out, torch.empty((T, m.read_out.shape[1]), dtype=torch.float32, device=m.device))


def law(logits, temperature):
    """Probabilities of the next token; temperature 0: all of it on the likeliest."""
    if temperature:
        return torch.softmax(logits / temperature, -1)
    return torch.zeros_like(logits).scatter_(-1, logits.argmax(-1, keepdim=True), 1.0)


def generate(target, draft, prompts, new, depth=4, branch=2, kind="same", page_size=16, temperature=1.0, seed=0):
    """At least `new` tokens behind each prompt; returns the texts, the tokens that stood in each step [steps, sequences] (0: the sequence waited), and the seconds of the steps."""
    B, dev = len(prompts), target.device
    parents = tree(depth, branch)
    n = len(parents)
    most = max(map(len, prompts)) + new + 2 * n + 2
    if not all(prompts) or most > len(target.positions):
        raise ValueError(f"prompts have 1 to {len(target.positions) - new - 2 * n - 2} tokens here")
    width = -(-most // page_size)
    both = [Sequences(m, B, B * width, page_size, width, kind) for m in (target, draft)]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def int32(x): return torch.tensor(x, dtype=torch.int32, device=dev)
    # the prompts but for their last tokens, which are the first trees' roots
    counts, total = int32([len(p) - 1 for p in prompts]), sum(map(len, prompts)) - B
    for s in both:
        slots, positions, starts = s.grow(counts, total)
        if total:
            s(torch.tensor([i for p in prompts for i in p[:-1]], device=dev), slots, positions, starts, None, max(map(len, prompts)) - 1)
    root = torch.tensor([p[-1] for p in prompts], device=dev)
    each = int32([n] * B)
    all_parents, starts = int32(parents * B), int32([n * b for b in range(B + 1)])
    masks = torch.empty((B * n, -(-n // 64)), dtype=torch.int64, device=dev)
    depths, positions = (torch.empty(B * n, dtype=torch.int32, device=dev) for _ in range(2))
    path, accepted = torch.empty((B, depth + 1), dtype=torch.int32, device=dev), torch.empty(B, dtype=torch.int32, device=dev)
    steps = []
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(new):                                                   # (a step brings one token at least)
        # ---- the draft: a level of the trees at a time, each level's drafts from their parents' rows
        t, d = both
        slots, _, _ = d.grow(each, B * n)
        nt.tree_masks(all_parents, starts, masks, depths, d.lengths, positions)
        ids, tokens = root[:, None].expand(B, n).clone(), torch.arange(B, device=dev)[:, None] * n
        drafts = torch.empty((B * n, target.read_out.shape[1]), dtype=torch.float32, device=dev)
        level = [0]
        while level:
            # (a level's tokens see their ancestors alone: their own rows of the masks, in a batch of their own)
            upto = level[-1] + 1
            rows = (tokens + torch.arange(upto, device=dev)).flatten()
            part = int32([upto * b for b in range(B + 1)])
            lengths, d.lengths = d.lengths, d.lengths - (n - upto)
            drafts[rows] = law(d(ids[:, :upto].flatten(), slots[rows], positions[rows], part, masks[rows], upto), temperature)
            d.lengths = lengths
            behind = [i for i, p in enumerate(parents) if p in level]
            for i in behind:
                row = drafts[tokens[:, 0] + parents[i]]
                ids[:, i] = torch.multinomial(row, 1, generator=gen)[:, 0] if temperature else row.argmax(-1)
            level = behind
        # ---- the target: the whole tree at once
        slots, _, _ = t.grow(each, B * n)
        rows = law(t(ids.flatten(), slots, positions, starts, masks, n), temperature)
        following = torch.empty(B, dtype=torch.int64, device=dev)
        full = t.lengths + (depth + 1) > most                               # no room for another tree behind this one: has its new tokens, and waits for the slower ones
        u, r = torch.rand(B * n, generator=gen, device=dev), torch.rand(B, generator=gen, device=dev)
        nt.verify_tree(rows, drafts, ids.flatten(), all_parents, starts, u, r, path, accepted, following, t.lengths, t.lengths)
        t.lengths.sub_(accepted * full)
        accepted.masked_fill_(full, 0)
        path.masked_fill_(full[:, None], -1)
        following = torch.where(full, root, following)
        d.lengths.copy_(t.lengths)
        for s in both:
            nt.cache_compact([c if c[2] is not None else c[:2] for c in s.model.cache], s.table, s.lengths, path, accepted)
        steps.append((path.clone(), ids, following.clone()))
        root = following
        if len(steps) * (depth + 1) >= new and min(sum(k) for k in zip(*[(p >= 0).sum(1).tolist() for p, _, _ in steps])) >= new:
            break
    torch.cuda.synchronize()
    seconds = time.perf_counter() - began
    texts, stood = [list(p) for p in prompts], []
    for p, ids, following in steps:
        stood.append((p >= 0).sum(1).tolist())
        for b in range(B):
            if stood[-1][b]:
                texts[b] += [ids[b, i].item() for i in p[b].tolist() if i > 0] + [following[b].item()]
    return texts, stood, seconds


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--cache", choices=["same", "e4m3", "int8"], default="same")
    p.add_argument("--temperature", type=float, default=1.0)
    for name, value in (("sequences", 8), ("prompt", 300), ("depth", 4), ("branch", 2), ("new", 64), ("seed", 0)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    target, draft = Decoder(seed=a.seed), Decoder(seed=a.seed)
    draft.layers = draft.layers[:1]
    g = torch.Generator().manual_seed(a.seed + 1)
    prompts = [torch.randint(len(target.tokens), (n,), generator=g).tolist() for n in torch.randint(1, a.prompt + 1, (a.sequences,), generator=g).tolist()]
    for new in (2, a.new):                                                 # (first calls load kernels and make the workspace)
        texts, stood, seconds = generate(target, draft, prompts, new, a.depth, a.branch, a.cache, temperature=a.temperature, seed=a.seed)
    kept = sum(map(sum, stood))
    print(f"{a.sequences} sequences, trees of {len(tree(a.depth, a.branch))}: {len(stood)} steps of {1e3 * seconds / len(stood):.2f} ms, {kept / len(stood) / a.sequences:.2f} tokens "
          f"of each sequence a step ({kept / seconds:.0f} tokens/s)")
    print("first text ends with", texts[0][-8:])


if __name__ == "__main__":
    main()
