"""The operators of a paged key / value cache, with inputs and plain forms: writing it (rounded to 16 bits or quantised to 8),
reading it back, and attention of new tokens over it.

Three kinds of case.  "write": new tokens into a cache of their own type, which is returned; into one of 8 bits they are read back in the
same pass, so that what comes back are the values that the codes and scales stand for.  "read": tokens of a cache back into dense
tensors.  "attend": a batch of sequences, each with its new tokens and a past of its own length.  Sizes are this repository's attention
workload (48 heads of 64) and generic ones with shared key heads.

A cache is [pages, page_size, heads, head_size] (`heads_first`: stored [pages, heads, page_size, head_size]); slot s is position
s % page_size of page s // page_size.  An 8-bit cache has a scale for each token and head."""
import math
import random

import torch

own = False

_DT = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}
_LARGEST = {"e4m3": 448.0, "i8": 127.0}
_BYTES = {"f16": 2, "bf16": 2, "e4m3": 1, "i8": 1}


def listed():
    return [
        # one new token of one sequence: latency is all there is to it
        dict(name="write_one", op="write", tokens=1, heads=8, size=128, page=16, heads_first=False, dtype="bf16", cache="e4m3"),
        # a decoding step of many sequences: a token each, scattered over the cache, in the tokens' own type
        dict(name="write_step", op="write", tokens=256, heads=48, size=64, page=16, heads_first=True, dtype="f16", cache="f16"),
        # whole prompts at once, quantised
        dict(name="write_prompts", op="write", tokens=16384, heads=8, size=128, page=64, heads_first=False, dtype="bf16", cache="i8"),
        # a short past of odd length, odd head count and head size, brought back to 16 bits
        dict(name="read_odd", op="read", tokens=777, heads=5, size=80, page=24, heads_first=False, dtype="f16", cache="e4m3"),
        # a long past brought back to 16 bits
        dict(name="read_long", op="read", tokens=65536, heads=8, size=128, page=64, heads_first=True, dtype="bf16", cache="e4m3"),
        # one sequence's next token after a short prompt: latency
        dict(name="decode_one", op="attend", batch=1, new=1, least=900, most=900, q_heads=48, heads=48, size=64, page=16, heads_first=False, window=0,
             dtype="f16", cache="f16"),
        # a decoding step of a serving batch, sequences of very different age, four query heads to a key head
        dict(name="decode_batch", op="attend", batch=64, new=1, least=17, most=4096, q_heads=32, heads=8, size=128, page=16, heads_first=False, window=0,
             dtype="bf16", cache="bf16"),
        # the same with a head of keys for each query head and a quantised cache
        dict(name="decode_own_heads", op="attend", batch=32, new=1, least=200, most=2047, q_heads=48, heads=48, size=64, page=32, heads_first=True, window=0,
             dtype="f16", cache="i8"),
        # two sequences over a very long quantised past: the keys have to be shared out
        dict(name="decode_long", op="attend", batch=2, new=1, least=100001, most=131072, q_heads=32, heads=8, size=128, page=64, heads_first=False, window=0,
             dtype="bf16", cache="e4m3"),
        # a ragged batch: single tokens beside chunks, an odd page size and head size, a sliding window
        dict(name="chunk_ragged", op="attend", batch=7, new=200, least=1, most=2500, q_heads=20, heads=5, size=80, page=24, heads_first=False, window=512,
             dtype="f16", cache="f16"),
        # whole prompts without a past: this repository's attention workload, causal
        dict(name="chunk_prompts", op="attend", batch=4, new=1024, least=1024, most=1024, q_heads=48, heads=48, size=64, page=64, heads_first=True, window=0,
             dtype="f16", cache="f16"),
        # a large chunk of one long prompt whose beginning is in the cache already
        dict(name="chunk_long", op="attend", batch=1, new=2048, least=18500, most=18500, q_heads=32, heads=8, size=128, page=64, heads_first=False, window=0,
             dtype="bf16", cache="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the ranges above: 1 to 32768 tokens written or read; 1 to 128 sequences of up to 131072 tokens, 1 to 2048 of them new."""
    dtype = rng.choice(["f16", "bf16"])
    c = dict(op=rng.choice(["write", "read", "attend", "attend", "attend"]), size=rng.choice([64, 64, 80, 96, 128, 128, 128, 256]),
             page=rng.choice([1, 16, 16, 24, 32, 64, 64, 128, 256]), heads_first=rng.random() < 0.5, dtype=dtype, cache=rng.choice([dtype, dtype, "e4m3", "i8"]))
    if c["op"] != "attend":
        c["heads"] = rng.choice([1, 2, 3, 5, 8, 16, 48])
        c["tokens"] = _log(rng, 1, min(32768, (1 << 26) // (c["heads"] * c["size"])))
        return c
    c["heads"] = rng.choice([1, 2, 4, 5, 8, 8, 16])
    c["q_heads"] = c["heads"] * rng.choice([1, 1, 3, 4, 4, 8, 16])
    if c["q_heads"] > 64:
        c["q_heads"] = c["heads"]
    if rng.random() < 0.5:
        c["new"], c["batch"] = rng.choice([1, 1, 1, 2, 4]), _log(rng, 1, 128)
        top = (1 << 27) // (c["batch"] * c["heads"] * c["size"])
    else:
        c["new"], c["batch"] = _log(rng, 8, 2048), _log(rng, 1, 8)
        top = min((1 << 27) // (c["batch"] * c["heads"] * c["size"]), (1 << 30) // (c["batch"] * c["q_heads"] * c["new"]))
    c["most"] = _log(rng, 1, max(1, min(131072, top)))
    c["least"] = rng.randint(1, c["most"])
    c["window"] = 0 if rng.random() < 0.75 else _log(rng, 1, 4096)
    return c


def _sequences(c):
    """(new tokens, length with them) of each sequence, the same for every seed: the first has the most of either."""
    rng = random.Random(c["batch"] * 1000003 + c["most"] * 101 + c["new"])
    lengths = [c["most"]] + [rng.randint(c["least"], c["most"]) for _ in range(c["batch"] - 1)]
    ragged = c["new"] > 4 and c["least"] < c["most"]
    new = [min(c["new"], lengths[0])] + [min(rng.randint(1, c["new"]) if ragged else c["new"], n) for n in lengths[1:]]
    return new, lengths


def work(c):
    per = c["heads"] * c["size"]
    scales = 8 * c["heads"] if c["cache"] in _LARGEST else 0                # of a token's keys and values
    if c["op"] != "attend":
        token = 2 * per * (2 + _BYTES[c["cache"]]) + scales + 8            # its 16-bit and its stored form, its slot
        return {"bytes": c["tokens"] * token * (2 if c["op"] == "write" and scales else 1), "flops": 0}
    new, lengths = _sequences(c)
    w = c["window"] or 1 << 40
    read = sum(min(n, w + m - 1) for m, n in zip(new, lengths))            # tokens of the cache that some query sees
    pairs = 0
    for m, n in zip(new, lengths):
        full = min(m, max(0, n - w + 1))                                   # queries with a whole window before them
        first = n - m + 1
        pairs += full * w + (m - full) * first + (m - full) * (m - full - 1) // 2 if full else m * first + m * (m - 1) // 2
    return {"bytes": read * (2 * per * _BYTES[c["cache"]] + scales) + sum(new) * c["q_heads"] * c["size"] * 4,
            "flops": 4 * pairs * c["q_heads"] * c["size"]}


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


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] != "attend":
        n = c["tokens"]
        pages = -(-n * 5 // 4 // c["page"]) + 1                             # a fifth of the cache is other sequences'
        s["slots"] = torch.randperm(pages * c["page"], generator=gen, device="cuda")[:n].contiguous()
        s["k"], s["v"] = (torch.randn((n, c["heads"], c["size"]), generator=gen, device="cuda").to(_DT[c["dtype"]]) for _ in range(2))
        s["cache"], s["scale"] = _shaped(c, pages, _DT[c["cache"]]) if c["op"] == "write" else _filled(c, pages, gen)
        return s
    new, lengths = _sequences(c)
    held = [-(-n // c["page"]) for n in lengths]
    s["cache"], s["scale"] = _filled(c, sum(held) + 3, gen)
    ids = torch.randperm(sum(held) + 3, generator=gen, device="cuda").to(torch.int32)
    s["table"] = torch.full((c["batch"], max(held)), -1, dtype=torch.int32, device="cuda")
    for b, (m, at) in enumerate(zip(held, [sum(held[:b]) for b in range(len(held))])):
        s["table"][b, :m] = ids[at:at + m]
    s["starts"] = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["max_new"], s["max_length"] = max(new), max(lengths)                  # what a program's scheduler knows on the host
    s["q"] = torch.randn((sum(new), c["q_heads"], c["size"]), generator=gen, device="cuda").to(_DT[c["dtype"]])
    s["out"] = torch.empty_like(s["q"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _held(cache, scale, page, at):
    """The tokens at position `at` of page `page`, in 32 bits."""
    x = cache.view(torch.uint8)[page, at].view(cache.dtype).float() if cache.element_size() == 1 else cache[page, at].float()
    return x if scale is None else x * scale[page, at][..., None]


def _quantised(x, kind):
    """Codes and scale of x: the scale is the largest magnitude over the type's largest value, in twelve significant bits, rounded up."""
    x = x.double()                                                          # (in 32 bits a quotient can fall on a border that it is beside)
    s = (x.abs().amax(-1) / _LARGEST[kind]).float()
    s = ((s.view(torch.int32) + 0xfff) & ~0xfff).view(torch.float32).clamp_min(2.0 ** -100)
    y = (x / s.double()[..., None]).float()
    return (y.round() if kind == "i8" else y).to(_DT[kind]), s


def _plain_write(s):
    c = s["case"]
    page, at = s["slots"] // c["page"], s["slots"] % c["page"]
    back = []
    for x, cache, scale in zip((s["k"], s["v"]), s["cache"], s["scale"]):
        if scale is None:
            cache[page, at] = x
        else:
            code, scale[page, at] = _quantised(x, c["cache"])
            cache.view(torch.uint8)[page, at] = code.view(torch.uint8)
            back.append(_held(cache, scale, page, at).to(x.dtype))
    return back + s["scale"] if back else s["cache"]


def _plain_read(s):
    c = s["case"]
    page, at = s["slots"] // c["page"], s["slots"] % c["page"]
    return [_held(cache, scale, page, at).to(_DT[c["dtype"]]) for cache, scale in zip(s["cache"], s["scale"])]


def _plain_attend(s):
    """Every sequence padded to the longest, the padding masked."""
    c, q, dev = s["case"], s["q"], s["q"].device
    group = c["q_heads"] // c["heads"]
    starts, lengths = s["starts"].long(), s["lengths"].long()
    count = starts[1:] - starts[:-1]
    row = torch.arange(s["max_new"], device=dev)
    real = row < count[:, None]                                             # [batch, new]
    token = torch.where(real, starts[:-1, None] + row, 0)
    pos = (lengths - count)[:, None] + row                                  # of each query
    key = torch.arange(s["max_length"], device=dev)
    inside = key < lengths[:, None]                                         # [batch, length]
    page = torch.where(inside, s["table"].long()[:, key // c["page"]], 0)
    k, v = (_held(t, u, page, key % c["page"]).permute(0, 2, 1, 3).contiguous() for t, u in zip(s["cache"], s["scale"]))     # [batch, heads, length, size]
    # queries that share a key head side by side: [batch, heads, new * group, size]
    x = q.float()[token].view(c["batch"], -1, c["heads"], group, c["size"]).permute(0, 2, 1, 3, 4).reshape(c["batch"], c["heads"], -1, c["size"])
    score = x @ k.transpose(2, 3).contiguous() * (1.0 / math.sqrt(c["size"]))
    seen = inside[:, None, :] & (key <= pos[..., None])
    if c["window"]:
        seen &= key > pos[..., None] - c["window"]
    seen = seen.repeat_interleave(group, 1)[:, None]
    score = score.masked_fill_(~seen, -math.inf)
    p = (score - score.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.where(total > 0, p @ v / total.clamp_min(1e-30), 0.0)
    o = o.view(c["batch"], c["heads"], -1, group, c["size"]).permute(0, 2, 1, 3, 4).reshape(c["batch"], -1, c["q_heads"], c["size"])
    return o[real].to(q.dtype)


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    c = s["case"]
    if not own:
        return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[c["op"]](s)
    import paper_2507_11978_amd as nt
    (kc, vc), (ks, vs) = s["cache"], s["scale"]
    if c["op"] == "write":
        nt.cache_write(s["k"], s["v"], s["slots"], kc, vc, ks, vs)
        if ks is None:
            return [kc, vc]
        k, v = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        nt.cache_read(kc, vc, s["slots"], k, v, ks, vs)
        return [k, v, ks, vs]
    if c["op"] == "read":
        k, v = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        nt.cache_read(kc, vc, s["slots"], k, v, ks, vs)
        return [k, v]
    return nt.sdpa_paged(s["q"], kc, vc, s["table"], s["starts"], s["lengths"], s["out"], ks, vs, window=c["window"], max_queries=s["max_new"],
                         max_length=s["max_length"])


# ------------------------------------------------------------------------------------------- in 64 bits
def _two_to(e):
    """2^e in 64 bits (torch.ldexp goes through a power in 32 bits, which is not exact on the GPU)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes(x, kind):
    """The values (64 bits) that x is quantised to, and the scales: borders by comparison in 64 bits, ties to the even code."""
    x = x.double()
    top = x.abs().amax(-1) / _LARGEST[kind]
    m, e = torch.frexp(top)
    s = (torch.ceil(m * 4096.0) * _two_to(e - 12)).clamp_min(2.0 ** -100)
    y = x / s[..., None]
    if kind == "i8":
        return torch.round(y) * s[..., None], s
    step = _two_to(torch.frexp(y.abs().clamp_min(2.0 ** -6))[1] - 4)       # three bits behind the leading one; 2^-9 below 2^-6
    return torch.round(y / step) * step * s[..., None], s


def exact(case, seed):
    c, s = case, prepare(case, seed)
    scales = s["scale"] if s["scale"][0] is not None else [None, None]
    full = lambda t, u: t.double() if u is None else t.double() * u.double()[..., None]  # noqa: E731
    if c["op"] == "write":
        flat = s["slots"]
        if scales[0] is None:
            want = []
            for x, cache in zip((s["k"], s["v"]), s["cache"]):
                y = cache.double().reshape(-1, c["heads"], c["size"])
                y[flat] = x.double()
                want.append(y.view(cache.shape))
            return want
        held, scale = zip(*[_exact_codes(x, c["cache"]) for x in (s["k"], s["v"])])
        for i in range(2):
            y = scales[i].double().reshape(-1, c["heads"])
            y[flat] = scale[i]
            scales[i] = y.view(scales[i].shape)
        return list(held) + scales
    if c["op"] == "read":
        return [full(t, u).reshape(-1, c["heads"], c["size"])[s["slots"]] for t, u in zip(s["cache"], scales)]
    group = c["q_heads"] // c["heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for b, (m, n) in enumerate(zip(*_sequences(c))):
        pages = s["table"][b, :-(-n // c["page"])].long()
        k, v = (full(t[pages], None if u is None else u[pages]).reshape(-1, c["heads"], c["size"])[:n] for t, u in zip(s["cache"], scales))
        pos = torch.arange(n - m, n, device="cuda")[:, None]
        key = torch.arange(n, device="cuda")
        hidden = key > pos
        if c["window"]:
            hidden = hidden | (key <= pos - c["window"])
        for h in range(c["q_heads"]):
            z = s["q"][at:at + m, h].double() @ k[:, h // group].t() / math.sqrt(c["size"])
            out[at:at + m, h] = torch.softmax(z.masked_fill(hidden, -math.inf), -1) @ v[:, h // group]
        at += m
    return out
