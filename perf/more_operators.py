"""The operators of decoding with drafted tokens over a paged key / value cache, with inputs and plain forms.

"fit": pages, slots and positions of a step's new tokens from the sequences' lengths.  "masks": a drafted tree's ancestors as bits, its depths and positions.
"attend": attention of every tree's tokens over the sequence's past and their own ancestors.  "verify": which drafted tokens stand, from the
target's (and the draft's) probabilities and given random numbers, and the token behind them.  "compact": the keys and values of the tokens that stand,
moved to the places behind the past, in every layer's cache.

A step's new tokens lie one sequence behind the other; token 0 of a sequence is the root of its tree (the last token that stands already), the others are
drafts, each behind its parent.  A cache is [pages, page_size, heads, head_size] (`heads_first`: stored [pages, heads, page_size, head_size]);
an 8-bit cache has a scale for each token and head.  Sizes are this repository's attention workload (48 heads of 64) and generic ones."""
import math
import random

import torch

own = False

_DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
_LARGEST = {"e4m3": 448.0, "i8": 127.0}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1, "i8": 1}


def listed():
    return [
        # a decoding step of a serving batch: a token to each sequence, a page to some
        dict(name="fit_step", op="fit", batch=256, least=17, most=4096, page=16, turnover=False, most_new=1),
        # sequences that ended give their pages back, and prompts of other requests take their places
        dict(name="fit_turnover", op="fit", batch=96, least=100, most=4000, page=32, turnover=True, most_new=2000),
        # one small tree of one sequence: latency is all there is to it
        dict(name="masks_one", op="masks", batch=1, new=8, most=900, window=0),
        # trees of many sequences, of different sizes, more nodes than one word has bits
        dict(name="masks_batch", op="masks", batch=128, new=100, most=4096, window=0),
        # a short draft of one sequence after a short prompt: latency
        dict(name="tree_one", op="attend", batch=1, new=8, least=900, most=900, q_heads=48, heads=48, size=64, page=16, heads_first=False, window=0,
             dtype="f16", cache="f16"),
        # a step of a serving batch, sequences of very different age, trees of 16 nodes, four query heads to a key head
        dict(name="tree_batch", op="attend", batch=32, new=16, least=17, most=4096, q_heads=32, heads=8, size=128, page=16, heads_first=False, window=0,
             dtype="bf16", cache="bf16"),
        # odd head size, page size and head count, ragged trees, a quantised cache, a sliding window
        dict(name="tree_ragged", op="attend", batch=16, new=26, least=1, most=3000, q_heads=20, heads=5, size=80, page=24, heads_first=True, window=2000,
             dtype="f16", cache="e4m3"),
        # two sequences over a very long quantised past, large trees
        dict(name="tree_long", op="attend", batch=2, new=64, least=100001, most=131072, q_heads=32, heads=8, size=128, page=64, heads_first=False, window=0,
             dtype="bf16", cache="i8"),
        # one sequence and a chain of drafts with their own probabilities: latency
        dict(name="verify_chain", op="verify", batch=1, new=6, vocabulary=32000, draft=True, chain=True, dtype="f32"),
        # a serving batch with trees
        dict(name="verify_batch", op="verify", batch=64, new=24, vocabulary=128000, draft=True, chain=False, dtype="f32"),
        # one sequence, a few tokens, a small model's layers
        dict(name="compact_one", op="compact", batch=1, new=8, most=900, layers=4, heads=4, size=64, page=16, heads_first=False, dtype="f16", cache="f16"),
        # a serving batch and many layers
        dict(name="compact_batch", op="compact", batch=64, new=32, most=300, layers=16, heads=8, size=128, page=16, heads_first=False, dtype="bf16", cache="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the ranges above: 1 to 512 sequences of up to 8192 tokens to fit; trees of 1 to 256 nodes; 1 to 64 trees of up to 128 nodes over up to
    131072 keys; vocabularies of 1000 to 160000; up to 16 layers to compact."""
    op = rng.choice(["fit", "masks", "attend", "attend", "attend", "verify", "verify", "compact"])
    if op == "fit":
        turnover = rng.random() < 0.5
        most = _log(rng, 16, 4000 if turnover else 8192)
        return dict(op=op, batch=_log(rng, 1, 96 if turnover else 512), least=rng.randint(1, most), most=most, page=rng.choice([1, 8, 16, 16, 24, 32, 64, 256]),
                    turnover=turnover, most_new=_log(rng, 1, 2000) if turnover else rng.choice([1, 1, 1, 7, 33]))
    if op == "masks":
        new = _log(rng, 1, 256)
        return dict(op=op, batch=_log(rng, 1, min(256, 16384 // new)), new=new, most=_log(rng, new, 8192), window=rng.choice([0, 0, 0, rng.randint(1, new)]))
    dtype = rng.choice(["f16", "bf16"])
    if op == "verify":
        vocabulary = _log(rng, 1000, 160000)
        batch = _log(rng, 1, 64)
        return dict(op=op, batch=batch, new=_log(rng, 1, max(1, min(48, 196000000 // (batch * vocabulary)))), vocabulary=vocabulary, draft=rng.random() < 0.6,
                    chain=rng.random() < 0.4, dtype=rng.choice(["f32", "f32", dtype]))
    c = dict(op=op, size=rng.choice([64, 64, 80, 96, 128, 128, 128, 256]), page=rng.choice([1, 16, 16, 24, 32, 64, 64, 128, 256]), heads_first=rng.random() < 0.5,
             dtype=dtype, cache=rng.choice([dtype, dtype, "e4m3", "i8"]), heads=rng.choice([1, 2, 4, 5, 8, 8, 16]))
    if op == "compact":
        c["layers"], c["new"] = rng.randint(1, 16), _log(rng, 2, 64)
        c["most"] = _log(rng, c["new"], 1000)
        c["batch"] = _log(rng, 1, max(1, min(64, 300000000 // ((c["most"] + c["page"]) * c["layers"] * c["heads"] * c["size"]))))
        return c
    c["q_heads"] = c["heads"] * rng.choice([1, 1, 3, 4, 4, 8, 16])
    if c["q_heads"] > 64:
        c["q_heads"] = c["heads"]
    c["batch"], c["new"] = _log(rng, 1, 64), _log(rng, 1, 128)
    top = min((1 << 27) // (c["batch"] * c["heads"] * c["size"]), (1 << 28) // (c["batch"] * c["q_heads"] * c["new"]))
    c["most"] = _log(rng, 1, max(1, min(131072, top)))
    c["least"] = rng.randint(1, c["most"])
    c["window"] = 0 if rng.random() < 0.75 else _log(rng, 1, 4096)
    return c


# ------------------------------------------------------------------------------------------------- the cases' shapes, the same for every seed
def _rng(c):
    return random.Random(c["batch"] * 1000003 + c.get("most", c.get("vocabulary", 0)) * 101 + c.get("new", 0))


def _sequences(c):
    """(new tokens, length with them) of each sequence: the first has the most of either."""
    rng = _rng(c)
    lengths = [c["most"]] + [rng.randint(min(c.get("least", c["most"] // 2), c["most"]), c["most"]) for _ in range(c["batch"] - 1)]
    ragged = c["op"] == "masks" or c.get("least", c["most"]) == 1
    new = [min(c["new"], lengths[0])] + [max(0, min(rng.randint(0, c["new"]) if ragged else c["new"], n)) for n in lengths[1:]]
    return new, [max(n, m) for n, m in zip(lengths, new)]


def _trees(c, new, rng):
    """A tree for each sequence: parents (-1: the root), each before its children, two or so to a node."""
    parents = []
    for n in new:
        parents += [-1 if i == 0 else i - 1 if c.get("chain") else rng.randint(max(0, (i - 1) // 3), max(0, (i - 1) // 2)) if rng.random() < 0.8 else rng.randint(0, i - 1)
                    for i in range(n)]
    return parents


def _ancestors(parents, new, window):
    """Bits of each token, as Python integers, and depths."""
    bits, depths, at = [], [], 0
    for n in new:
        for i in range(n):
            j, d, b = i, 0, 0
            while j >= 0:
                b |= (1 << j) if not window or d < window else 0
                j, d = parents[at + j], d + 1
            bits.append(b)
            depths.append(d - 1)
        at += n
    return bits, depths


def _signed(x):
    return x - (1 << 64) if x >> 63 else x


def _requests(c):
    """Of each sequence: its length now, its length before (its pages are of that), its new tokens."""
    rng = _rng(c)
    before = [c["most"]] + [rng.randint(c["least"], c["most"]) for _ in range(c["batch"] - 1)]
    ended = [c["turnover"] and rng.random() < 0.5 for _ in before]
    if c["turnover"]:
        ended[0] = True
    now = [0 if e else n for e, n in zip(ended, before)]
    new = [rng.randint(1, c["most_new"]) if e or not c["turnover"] else 1 for e in ended]
    return now, before, new


def _accepted(c):
    """Of each sequence: its new tokens, its past's length, and which of the new ones stand (the first does; no place that is written is read)."""
    rng = _rng(c)
    new, lengths = [], []
    paths = []
    for _ in range(c["batch"]):
        n = c["new"]
        count = rng.randint(1, max(1, min(6, n // 2)))
        new.append(n)
        lengths.append(rng.randint(max(n, c["most"] // 2), c["most"]))
        paths.append([0] + sorted(rng.sample(range(count, n), count - 1)) if count > 1 else [0])
    return new, [m - n for m, n in zip(lengths, new)], paths


def work(c):
    if c["op"] == "fit":
        now, before, new = _requests(c)
        held = lambda n: -(-n // c["page"])  # noqa: E731
        moved = sum(abs(held(n + m) - held(n)) for n, m in zip(now, new)) + (sum(held(n + m) for n, m in zip(now, new) if n == 0) if c["turnover"] else 0)
        return {"bytes": (2 if c["turnover"] else 1) * c["batch"] * 28 + 8 * moved + 12 * sum(new), "flops": 0}
    if c["op"] == "masks":
        new, _ = _sequences(c)
        return {"bytes": sum(new) * (12 + 8 * (-(-max(new) // 64))) + 8 * c["batch"], "flops": 0}
    if c["op"] == "verify":
        # the row in which the walk ends, the draft's with it where there is one
        rows = 2 if c["draft"] else 1
        return {"bytes": c["batch"] * c["vocabulary"] * _BYTES[c["dtype"]] * rows + c["batch"] * c["new"] * 32, "flops": 2 * c["batch"] * c["vocabulary"]}
    per = c["heads"] * c["size"]
    scales = 8 * c["heads"] if c["cache"] in _LARGEST else 0                # of a token's keys and values
    if c["op"] == "compact":
        moved = sum(sum(i != k for k, i in enumerate(p)) for p in _accepted(c)[2])
        return {"bytes": 2 * moved * c["layers"] * (2 * per * _BYTES[c["cache"]] + scales) + c["batch"] * 32, "flops": 0}
    new, lengths = _sequences(c)
    bits, depths = _ancestors(_trees(c, new, _rng(c)), new, c["window"])
    w = c["window"] or 1 << 40
    read = sum(min(n, w + m - 1) for m, n in zip(new, lengths))            # tokens of the cache that some query sees
    pairs, at = 0, 0
    for m, n in zip(new, lengths):
        pairs += sum(min(n - m, max(0, w - 1 - depths[at + i])) + bin(bits[at + i]).count("1") for i in range(m))
        at += m
    return {"bytes": read * (2 * per * _BYTES[c["cache"]] + scales) + sum(new) * (c["q_heads"] * c["size"] * 4 + 8), "flops": 4 * pairs * c["q_heads"] * c["size"]}


def _shaped(c, pages, dtype):
    """An empty cache, and its scales if it has any."""
    shape = (pages, c["heads"], c["page"], c["size"]) if c["heads_first"] else (pages, c["page"], c["heads"], c["size"])
    cache = [torch.zeros(shape, dtype=dtype, device="cuda") for _ in range(2)]
    scale = [torch.ones(shape[:3], dtype=torch.float32, device="cuda") if c["cache"] in _LARGEST else None for _ in range(2)]
    if c["heads_first"]:
        cache, scale = [t.transpose(1, 2) for t in cache], [s if s is None else s.transpose(1, 2) for s in scale]
    return cache, scale


def _filled(c, pages, gen):
    """A cache of tokens of everyday size."""
    if c["cache"] not in _LARGEST:
        return [t.copy_(torch.randn(t.shape, generator=gen, device="cuda")) for t in _shaped(c, pages, _DT[c["cache"]])[0]], [None, None]
    cache, scale = _shaped(c, pages, _DT[c["cache"]])
    for t, s in zip(cache, scale):
        x = torch.randn(t.shape, generator=gen, device="cuda")
        s.copy_(x.abs().amax(-1) / _LARGEST[c["cache"]])
        x = x / s[..., None]
        t.copy_(x.round().clamp(-127, 127) if c["cache"] == "i8" else x.clamp(-448, 448))
    return cache, scale


def _int(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def _paged(s, c, lengths, gen):
    """Pages in random order for sequences of these lengths: how many there are."""
    held = [-(-n // c["page"]) for n in lengths]
    ids = torch.randperm(sum(held) + 3, generator=gen, device="cuda").to(torch.int32)
    s["table"] = torch.full((c["batch"], max(held)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, m in enumerate(held):
        s["table"][b, :m] = ids[at:at + m]
        at += m
    return sum(held) + 3


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "fit":
        now, before, new = _requests(c)
        width = -(-(max(max(n + m for n, m in zip(now, new)), max(before)) + 64) // c["page"])
        held = [-(-n // c["page"]) for n in before]
        spare = sum(-(-(n + m) // c["page"]) for n, m in zip(now, new)) + 8
        ids = torch.randperm(sum(held) + spare, generator=gen, device="cuda").to(torch.int32)
        place = _int([b * width + e for b, m in enumerate(held) for e in range(m)], torch.int64)
        s["table"] = torch.full((c["batch"] * width,), -1, dtype=torch.int32, device="cuda").index_put_((place,), ids[:sum(held)]).view(c["batch"], width)
        s["free"] = torch.cat([ids[sum(held):], torch.full((sum(held),), -1, dtype=torch.int32, device="cuda")])
        s["free_count"], s["held"] = _int([spare]), _int(held)
        s["lengths"], s["counts"], s["none"] = _int(now), _int(new), _int([0] * len(new))
        s["starts"], s["new_lengths"] = _int([0] * (c["batch"] + 1)), _int([0] * c["batch"])
        s["slots"] = torch.full((sum(new),), -1, dtype=torch.int64, device="cuda")
        s["positions"] = torch.zeros(sum(new), dtype=torch.int32, device="cuda")
        return s
    if c["op"] == "verify":
        new = [c["new"]] * c["batch"]
        parents = _trees(c, new, random.Random(seed))
        T, V = sum(new), c["vocabulary"]
        at = _int([(t // c["new"]) * c["new"] + max(0, p) for t, p in enumerate(parents)], torch.int64)
        # a target that is sure of itself in places, a draft that is near it; each draft is drawn from the draft's row of its parent
        s["target"] = torch.empty((T, V), dtype=_DT[c["dtype"]], device="cuda")
        draft = torch.empty((T, V), dtype=_DT[c["dtype"]], device="cuda")
        ids = torch.zeros(T, dtype=torch.int64, device="cuda")
        for lo in range(0, T, 256):
            x = torch.randn((min(256, T - lo), V), generator=gen, device="cuda") * 3.0
            s["target"][lo:lo + 256] = torch.softmax(x, -1)
            draft[lo:lo + 256] = torch.softmax(x + torch.randn(x.shape, generator=gen, device="cuda") * 0.7, -1)
        for lo in range(0, T, 256):
            ids[lo:lo + 256] = torch.multinomial(draft[at[lo:lo + 256]].float(), 1, generator=gen)[:, 0]
        s["draft"], s["ids"], s["parents"] = draft if c["draft"] else None, ids, _int(parents)
        s["starts"] = _int([i * c["new"] for i in range(c["batch"] + 1)])
        s["uniform"] = torch.rand(T, generator=gen, device="cuda")
        s["last_uniform"] = torch.rand(c["batch"], generator=gen, device="cuda")
        s["lengths"] = torch.randint(c["new"], 4096, (c["batch"],), generator=gen, device="cuda").to(torch.int32)
        s["new_lengths"], s["accepted"] = torch.zeros_like(s["lengths"]), torch.zeros_like(s["lengths"])
        s["path"] = torch.zeros((c["batch"], min(c["new"], 8)), dtype=torch.int32, device="cuda")
        s["next"] = torch.zeros(c["batch"], dtype=torch.int64, device="cuda")
        return s
    if c["op"] == "compact":
        new, past, paths = _accepted(c)
        pages = _paged(s, c, [n + m for n, m in zip(past, new)], gen)
        filled = [_filled(c, pages, gen) for _ in range(c["layers"])]
        s["caches"] = [(k, v) if ks is None else (k, v, ks, vs) for (k, v), (ks, vs) in filled]
        width = max(map(len, paths))
        s["path"] = _int([p + [-1] * (width - len(p)) for p in paths])
        s["accepted"], s["lengths"] = _int([len(p) for p in paths]), _int([n + len(p) for n, p in zip(past, paths)])
        return s
    new, lengths = _sequences(c)
    s["starts"], s["lengths"] = _int([sum(new[:b]) for b in range(len(new) + 1)]), _int(lengths)
    s["max_new"], s["max_length"] = max(new), max(lengths)                  # what a program's scheduler knows on the host
    words = -(-max(new) // 64)
    if c["op"] == "masks":
        s["parents"] = _int(_trees(c, new, random.Random(seed)))
        T = sum(new)
        s["masks"] = torch.zeros((T, words), dtype=torch.int64, device="cuda")
        s["depths"], s["positions"] = (torch.zeros(T, dtype=torch.int32, device="cuda") for _ in range(2))
        return s
    s["cache"], s["scale"] = _filled(c, _paged(s, c, lengths, gen), gen)
    bits, depths = _ancestors(_trees(c, new, random.Random(seed)), new, c["window"])
    s["masks"] = _int([[_signed((b >> (64 * w)) & ((1 << 64) - 1)) for w in range(words)] for b in bits], torch.int64)
    s["depths"] = _int(depths)
    s["q"] = torch.randn((sum(new), c["q_heads"], c["size"]), generator=gen, device="cuda").to(_DT[c["dtype"]])
    s["out"] = torch.empty_like(s["q"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_fit_once(s, counts, tokens):
    """Pages given back from the last sequence's last to the first's first, then taken by the first sequence's first missing entry, and so on."""
    page, table, held, free = s["case"]["page"], s["table"], s["held"].long(), s["free"]
    B, width = table.shape
    dev = table.device
    starts = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), counts.long().cumsum(0)])
    s["new_lengths"].copy_(s["lengths"] + counts)
    want = ((s["new_lengths"].long() + page - 1) // page).clamp_max(width)[:, None]
    entry = torch.arange(width, device=dev)
    surplus, missing = (entry >= want) & (entry < held[:, None]), (entry >= held[:, None]) & (entry < want)
    number, taken = surplus.flatten().long().cumsum(0).view(B, width), missing.flatten().long().cumsum(0).view(B, width)
    top = s["free_count"].long().clamp_min(0) + number[-1, -1]
    longer = torch.cat([free, free[:1]])                                    # (one place more, for what is not given back)
    longer[torch.where(surplus, top - number, free.numel())] = table
    free.copy_(longer[:-1])
    at = top - taken
    got = missing & (at >= 0)
    table.copy_(torch.where(got, free[at.clamp(0, free.numel() - 1)], torch.where(missing, -1, table)))
    held = torch.minimum(held, want[:, 0]) + got.sum(1)
    s["held"].copy_(held)
    s["free_count"].copy_(top - taken[-1, -1])
    s["starts"].copy_(starts)
    if tokens:
        t = torch.arange(s["slots"].numel(), device=dev)
        b = torch.searchsorted(starts[1:].contiguous(), t, right=True).clamp_max(B - 1)
        pos = s["lengths"].long()[b] + t - starts[b]
        e = pos // page
        here = (t < starts[-1]) & (e < held[b])
        s["slots"].copy_(torch.where(here, table[b, e.clamp(0, width - 1)].long() * page + pos % page, -1))
        s["positions"].copy_(torch.where(t < starts[-1], pos, 0))


def _plain_fit(s):
    if s["case"]["turnover"]:
        _plain_fit_once(s, s["none"], False)
    _plain_fit_once(s, s["counts"], True)


def _plain_masks(s):
    """The ancestors' relation doubled until it is closed: who is seen over at most 1, 2, 4 ... edges (a window: those too far up are left out again)."""
    c, dev = s["case"], s["parents"].device
    starts = s["starts"].long()
    count = starts[1:] - starts[:-1]
    n, words = s["max_new"], s["masks"].shape[1]
    row = torch.arange(n, device=dev)
    real = row < count[:, None]
    token = torch.where(real, starts[:-1, None] + row, 0)
    parent = torch.where(real, s["parents"].long()[token], -1)
    reach = (parent[..., None] == row).float() + torch.eye(n, device=dev)
    for _ in range(max(1, n - 1).bit_length()):
        reach = ((reach @ reach) > 0).float()
    depth = reach.sum(-1).long() - 1
    seen = reach > 0
    if c["window"]:
        seen = seen & (depth[:, None, :] > depth[:, :, None] - c["window"])
    seen = torch.nn.functional.pad(seen, (0, 64 * words - n)).view(len(count), n, words, 64)
    masks = (seen.long() << torch.arange(64, device=dev)).sum(-1)
    past = (s["lengths"].long() - count)[:, None] + depth
    s["masks"].copy_(masks[real])
    s["depths"].copy_(depth[real])
    s["positions"].copy_(past[real])


def _held(cache, scale, page, at):
    """The tokens at position `at` of page `page`, in 32 bits."""
    x = cache.view(torch.uint8)[page, at].view(cache.dtype).float() if cache.element_size() == 1 else cache[page, at].float()
    return x if scale is None else x * scale[page, at][..., None]


def _plain_attend(s):
    """Every sequence padded to the longest, the padding masked."""
    c, q, dev = s["case"], s["q"], s["q"].device
    group = c["q_heads"] // c["heads"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    count = starts[1:] - starts[:-1]
    row = torch.arange(s["max_new"], device=dev)
    real = row < count[:, None]                                             # [batch, new]
    token = torch.where(real, starts[:-1, None] + row, 0)
    past = (lengths - count)[:, None]
    key = torch.arange(s["max_length"], device=dev)
    inside = key < lengths[:, None]                                         # [batch, length]
    page = torch.where(inside, s["table"].long()[:, key // c["page"]], 0)
    k, v = (_held(t, u, page, key % c["page"]).permute(0, 2, 1, 3).contiguous() for t, u in zip(s["cache"], s["scale"]))     # [batch, heads, length, size]
    # queries that share a key head side by side: [batch, heads, new * group, size]
    x = q.float()[token].view(c["batch"], -1, c["heads"], group, c["size"]).permute(0, 2, 1, 3, 4).reshape(c["batch"], c["heads"], -1, c["size"])
    score = x @ k.transpose(2, 3).contiguous() * (1.0 / math.sqrt(c["size"]))
    own_key = key - past                                                    # [batch, length], its number among the new tokens
    word = s["masks"][token]                                                # [batch, new, words]
    bit = (torch.gather(word, 2, (own_key.clamp(0, s["max_new"] - 1) // 64)[:, None, :].expand(-1, s["max_new"], -1)) >> (own_key.clamp_min(0) % 64)[:, None, :]) & 1
    seen = torch.where((own_key < 0)[:, None, :], True, bit == 1) & inside[:, None, :]
    if c["window"]:
        seen &= (own_key >= 0)[:, None, :] | (own_key[:, None, :] > s["depths"].long()[token][..., None] - c["window"])
    seen = seen.repeat_interleave(group, 1)[:, None]
    score = score.masked_fill_(~seen, -math.inf)
    p = (score - score.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, p @ v / total.clamp_min(1e-30), 0.0)
    o = o.view(c["batch"], c["heads"], -1, group, c["size"]).permute(0, 2, 1, 3, 4).reshape(c["batch"], -1, c["q_heads"], c["size"])
    return o[real].to(q.dtype)


def _plain_verify(s):
    """The drafts in their order, of all sequences at a time: a node's children come behind it, so that one pass is the walk."""
    c, dev = s["case"], s["ids"].device
    starts = s["starts"].long()
    count = starts[1:] - starts[:-1]
    B, width = s["path"].shape
    at = torch.arange(B, device=dev)
    node = torch.zeros(B, dtype=torch.int64, device=dev)
    w = s["target"][starts[:-1]].double()                                   # (borders between tokens are compared: 64 bits)
    m = torch.ones(B, dtype=torch.float64, device=dev)
    path = torch.full((B, width + 1), -1, dtype=torch.int64, device=dev)
    path[:, 0] = 0
    accepted = torch.ones(B, dtype=torch.int64, device=dev)
    for i in range(1, c["new"]):
        t = starts[:-1] + i
        child = (i < count) & (s["parents"][t] == node) & (accepted < width)
        x = s["ids"][t]
        of_x = w[at, x]
        q = s["draft"][starts[:-1] + node, x].double() if c["draft"] else 1.0
        good = child & (s["uniform"][t].double() * q * m < of_x)
        bad = child & ~good
        if c["draft"]:
            left = torch.where(m[:, None] > 0, w / m.clamp_min(1e-300)[:, None] - s["draft"][starts[:-1] + node].double(), 0.0).clamp_min(0.0)
            w = torch.where(bad[:, None], left, w)
            m = torch.where(bad, left.sum(1), m)
        else:
            w[at, x] = torch.where(bad, 0.0, of_x)
            m = torch.where(bad, (m - of_x).clamp_min(0.0), m)
        w = torch.where(good[:, None], s["target"][t].double(), w)
        m = torch.where(good, 1.0, m)
        path[at, torch.where(good, accepted, width)] = i
        node = torch.where(good, i, node)
        accepted = accepted + good
    none = w.sum(1, keepdim=True) <= 0
    w = torch.where(none, s["target"][starts[:-1] + node].double(), w)
    upto = w.cumsum(1)
    s["next"].copy_((upto <= s["last_uniform"].double()[:, None] * upto[:, -1:]).sum(1).clamp_max(c["vocabulary"] - 1))
    s["path"].copy_(path[:, :-1])
    s["accepted"].copy_(accepted)
    s["new_lengths"].copy_(s["lengths"] - count + accepted)


def _plain_compact(s):
    c = s["case"]
    width = s["path"].shape[1]
    order = torch.arange(width, device=s["path"].device)
    stands = order < s["accepted"][:, None]
    past = (s["lengths"] - s["accepted"]).long()[:, None]
    here, there = past + torch.where(stands, s["path"].long(), 0), past + torch.where(stands, order, 0)       # (the others: the root onto itself)
    places = [(torch.gather(s["table"].long(), 1, p // c["page"]), p % c["page"]) for p in (here, there)]
    for cache in s["caches"]:
        for t in cache:
            t = t.view(torch.uint8) if t.element_size() == 1 else t
            t[places[1]] = t[places[0]]


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if own:
        import paper_2507_11978_amd as nt
    if c["op"] == "fit":
        if own:
            pool = (s["table"], s["held"], s["free"], s["free_count"], s["starts"], s["new_lengths"])
            if c["turnover"]:
                nt.cache_fit(s["lengths"], s["none"], c["page"], *pool, s["slots"][:0], s["positions"][:0])
            nt.cache_fit(s["lengths"], s["counts"], c["page"], *pool, s["slots"], s["positions"])
        else:
            _plain_fit(s)
        return [s[n] for n in ("starts", "new_lengths", "slots", "positions", "table", "held", "free", "free_count")]
    if c["op"] == "masks":
        if own:
            nt.tree_masks(s["parents"], s["starts"], s["masks"], s["depths"], s["lengths"], s["positions"], window=c["window"])
        else:
            _plain_masks(s)
        return [s["masks"], s["depths"], s["positions"]]
    if c["op"] == "attend":
        if not own:
            return _plain_attend(s)
        (kc, vc), (ks, vs) = s["cache"], s["scale"]
        return nt.sdpa_paged_tree(s["q"], kc, vc, s["table"], s["starts"], s["lengths"], s["masks"], s["out"], ks, vs, depths=s["depths"] if c["window"] else None,
                                  window=c["window"], max_queries=s["max_new"], max_length=s["max_length"])
    if c["op"] == "verify":
        if own:
            nt.verify_tree(s["target"], s["draft"], s["ids"], s["parents"], s["starts"], s["uniform"], s["last_uniform"], s["path"], s["accepted"], s["next"],
                           s["lengths"], s["new_lengths"])
        else:
            _plain_verify(s)
        return [s["path"], s["accepted"], s["next"], s["new_lengths"]]
    if own:
        nt.cache_compact(s["caches"], s["table"], s["lengths"], s["path"], s["accepted"])
    else:
        _plain_compact(s)
    if c["cache"] not in _LARGEST:
        return [t for cache in s["caches"] for t in cache]
    return [t.float() * u[..., None] for k, v, ks, vs in s["caches"] for t, u in ((k, ks), (v, vs))]         # (what the codes stand for)


# ------------------------------------------------------------------------------------------- in 64 bits
def _exact_fit(s):
    """Lists, one sequence after the other."""
    c = s["case"]
    table, held, free, top = s["table"].tolist(), s["held"].tolist(), s["free"].tolist(), s["free_count"].item()
    lengths, counts = s["lengths"].tolist(), s["counts"].tolist()
    slots, positions, starts = [], [], [0]
    for adding in ([[0] * len(counts)] if c["turnover"] else []) + [counts]:
        after = [n + m for n, m in zip(lengths, adding)]
        want = [-(-n // c["page"]) for n in after]
        for b in reversed(range(len(want))):
            while held[b] > want[b]:
                held[b] -= 1
                free[top] = table[b][held[b]]
                top += 1
        for b in range(len(want)):
            while held[b] < want[b]:
                top -= 1
                table[b][held[b]] = free[top]
                held[b] += 1
    for b, (n, m) in enumerate(zip(lengths, counts)):
        positions += range(n, n + m)
        slots += [table[b][p // c["page"]] * c["page"] + p % c["page"] for p in range(n, n + m)]
        starts.append(starts[-1] + m)
    return [_int(x, torch.int64) for x in (starts, after, slots, positions, table, held, free, [top])]


def _exact_verify(s):
    """A sequence at a time, node by node."""
    c = s["case"]
    parents, ids, u, last = s["parents"].tolist(), s["ids"].tolist(), s["uniform"].tolist(), s["last_uniform"].tolist()
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    width = s["path"].shape[1]
    paths, accepted, following, after = [], [], [], []
    for b in range(c["batch"]):
        lo, hi = starts[b], starts[b + 1]
        path, w, m = [0], s["target"][lo].double(), 1.0
        walking = True
        while walking and len(path) < width:
            walking = False
            node = path[-1]
            q = s["draft"][lo + node].double() if c["draft"] else None
            for t in range(lo + node + 1, hi):
                if parents[t] != node:
                    continue
                of_x = w[ids[t]].item()
                if u[t] * (1.0 if q is None else q[ids[t]].item()) * m < of_x:
                    path.append(t - lo)
                    w, m, walking = s["target"][t].double(), 1.0, True
                    break
                if q is None:
                    w[ids[t]] = 0.0
                    m = max(0.0, m - of_x)
                elif m > 0:
                    w = (w / m - q).clamp(min=0.0)
                    m = w.sum().item()
        if w.sum() <= 0:
            w = s["target"][lo + path[-1]].double()
        upto = torch.cumsum(w, 0)
        following.append(min(c["vocabulary"] - 1, torch.searchsorted(upto, last[b] * upto[-1], right=True).item()))
        paths.append(path + [-1] * (width - len(path)))
        accepted.append(len(path))
        after.append(lengths[b] - (hi - lo) + len(path))
    return [_int(x, torch.int64) for x in (paths, accepted, following, after)]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "fit":
        return _exact_fit(s)
    if c["op"] == "verify":
        return _exact_verify(s)
    if c["op"] == "masks":
        new, lengths = _sequences(c)
        bits, depths = _ancestors(s["parents"].tolist(), new, c["window"])
        past = [n - m for m, n in zip(new, lengths) for _ in range(m)]
        return [_int([[_signed((b >> (64 * w)) & ((1 << 64) - 1)) for w in range(s["masks"].shape[1])] for b in bits], torch.int64), _int(depths, torch.int64),
                _int([p + d for p, d in zip(past, depths)], torch.int64)]
    if c["op"] == "compact":
        out, (_, pasts, paths) = [], _accepted(c)
        for cache in s["caches"]:
            for x, u in zip(cache[:2], cache[2:] or (None, None)):
                x = x.double() if u is None else x.double() * u.double()[..., None]
                for row, past, path in zip(s["table"].tolist(), pasts, paths):
                    for k, i in enumerate(path):
                        f, t = past + i, past + k
                        x[row[t // c["page"]], t % c["page"]] = x[row[f // c["page"]], f % c["page"]].clone()
                out.append(x)
        return out
    group = c["q_heads"] // c["heads"]
    full = lambda t, u: t.double() if u is None else t.double() * u.double()[..., None]  # noqa: E731
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    new, lengths = _sequences(c)
    bits, depths = _ancestors(_trees(c, new, random.Random(seed)), new, c["window"])
    at = 0
    for b, (m, n) in enumerate(zip(new, lengths)):
        if m == 0:
            continue
        pages = s["table"][b, :-(-n // c["page"])].long()
        k, v = (full(t[pages], None if u is None else u[pages]).reshape(-1, c["heads"], c["size"])[:n] for t, u in zip(s["cache"], s["scale"]))
        hidden = torch.zeros((m, n), dtype=torch.bool)
        for i in range(m):
            if c["window"]:
                hidden[i, :max(0, min(n - m, n - m + depths[at + i] - c["window"] + 1))] = True
            for j in range(m):
                hidden[i, n - m + j] = not (bits[at + i] >> j) & 1
        hidden = hidden.cuda()
        for h in range(c["q_heads"]):
            z = s["q"][at:at + m, h].double() @ k[:, h // group].t() / math.sqrt(c["size"])
            out[at:at + m, h] = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ v[:, h // group]
        at += m
    return out
