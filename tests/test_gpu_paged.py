"""GPU parity of the paged key / value cache (cache_write, cache_read, sdpa_paged) against the fp64 oracle.

Writing and reading are exact: codes and scales are integers and short numbers that either side computes alike, a value read is one rounding
of code * scale, so all of it is compared bit by bit.

Attention.  With h = eps / 2 of the 16-bit type and A = sum_j p_j |V_j| of an output (64 bits): rounding a weight changes its term by h, at most h A in
all; the sum of the rounded weights is off by h, h |O| <= h A; rounding the result adds h |O| <= h A (and h^2 terms: 1 %).  Scores are fp32 sums of `size`
products of exact factors, 2^-24 (size + 8) of the sum of their magnitudes, which for the inputs used is at most 4 (1 + largest |score|) sqrt(size) (unit
normal vectors); a score's error is its weight's relative error.  fp16 weights below 2^-14 of the reference round to multiples of 2^-24 (half
a step each: 2^-25 of it, twice that where a scale is folded in), for each of the keys, against values of at most max |V|."""
import numpy as np
import pytest
import torch

import paper_2507_11978_amd as nt
from oracle import paged as op

pytestmark = pytest.mark.gpu
TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "i8": torch.int8}


def normal(shape, dt, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(TORCH[dt])


def f64(t):
    return t.double().cpu().numpy() if t.dtype not in (torch.float8_e4m3fn,) else t.float().double().cpu().numpy()


def raw(t):
    """bits, for comparing"""
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]).cpu()


def empty_cache(pages, page, heads, size, kind, layout="dense", fill=0):
    """K, V (and scales) of a cache of the type `kind`; every byte of it `fill`."""
    def one(shape, dt):
        n = 1
        for s in shape:
            n *= s
        if layout == "heads first":
            shape = (shape[0], shape[2], shape[1]) + tuple(shape[3:])
        if layout == "padded" and len(shape) == 4:               # a row inside longer rows, starting off any boundary
            es = torch.empty((), dtype=dt).element_size()
            buf = torch.full((n // shape[3] * (shape[3] + 3) * es + 64 * es,), fill, dtype=torch.uint8, device="cuda").view(dt)
            return buf[3:3 + n // shape[3] * (shape[3] + 3)].view(*shape[:3], shape[3] + 3)[..., :shape[3]]
        t = torch.full((n * torch.empty((), dtype=dt).element_size(),), fill, dtype=torch.uint8, device="cuda").view(dt).view(shape)
        return t.transpose(1, 2) if layout == "heads first" else t
    k, v = (one((pages, page, heads, size), TORCH[kind]) for _ in range(2))
    if kind in op.LARGEST:
        ks, vs = (one((pages, page, heads), torch.float32) for _ in range(2))
        return k, v, ks, vs
    return k, v, None, None


# ------------------------------------------------------------------------------------------ writing, reading
@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["same", "e4m3", "i8"])
@pytest.mark.parametrize("tokens,heads,size,page,layout", [(1, 1, 8, 1, "dense"), (1, 8, 128, 16, "dense"), (37, 3, 64, 7, "heads first"), (50, 5, 80, 24, "padded"),
                                                           (33, 2, 256, 16, "dense"), (19, 3, 136, 5, "heads first"), (300, 48, 64, 32, "padded")])
def test_write_and_read_back(dt, kind, tokens, heads, size, page, layout):
    kind = dt if kind == "same" else kind
    pages = -(-tokens * 3 // 2 // page) + 1
    k, v = normal((tokens, heads, size), dt, 1), normal((tokens, heads, size), dt, 2, 37.0)
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(3))[:tokens]
    c = empty_cache(pages, page, heads, size, kind, layout, fill=0x5a)
    before = [None if t is None else raw(t) for t in c]
    nt.cache_write(k.cuda(), v.cuda(), slots.cuda(), *c)
    torch.cuda.synchronize()
    P, at = slots // page, slots % page
    for x, cache, scale, was, was_scale in zip((k, v), c[:2], c[2:], before[:2], before[2:]):
        got = raw(cache)
        if scale is None:
            assert torch.equal(got[P, at], raw(x))
        else:
            code, s = op.quantise(f64(x), kind, dt)
            held = P.numpy(), at.numpy()
            assert np.array_equal(f64(cache)[held], code) and np.array_equal(f64(scale)[held], s)
            assert torch.equal(raw(scale).index_put((P, at), was_scale[P, at]), was_scale)
        assert torch.equal(got.index_put((P, at), was[P, at]), was)          # nothing else was touched
    # back, some slots twice, some of no cache; into rows of a wider tensor
    again = torch.cat([slots, slots[:5], torch.tensor([-1, pages * page, -2 ** 62, 2 ** 62])])
    out = [torch.full((len(again), heads, size + 5), 7.0, dtype=TORCH[dt], device="cuda") for _ in range(2)]
    nt.cache_read(c[0], c[1], again.cuda(), out[0][..., 2:2 + size], out[1][..., 2:2 + size], c[2], c[3])
    torch.cuda.synchronize()
    for x, o in zip((k, v), out):
        if kind == dt:
            want = x
        else:
            code, s = op.quantise(f64(x), kind, dt)
            want = torch.from_numpy(code * s[..., None]).to(torch.float32).to(TORCH[dt])
        want = torch.cat([want, want[:5], torch.zeros(4, heads, size, dtype=TORCH[dt])])
        assert torch.equal(o[..., 2:2 + size].cpu(), want)
        assert (o[..., :2] == 7).all() and (o[..., 2 + size:] == 7).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
def test_rows_where_quantising_can_go_wrong(dt, kind):
    L, size, n = op.LARGEST[kind], 64, 4000
    g = torch.Generator().manual_seed(11)
    x = torch.randn((n, 1, size), generator=g)
    # borders: whole multiples of half a step of a scale that the row's largest value fixes, as near as 16 bits come to them, and the neighbours
    scale = (torch.rand((n // 2, 1, 1), generator=g) + 0.5).to(TORCH[dt]).float()
    half = torch.randint(0, int(2 * L), (n // 2, 1, size), generator=g) / 2.0 if kind == "i8" else torch.from_numpy((op.E4M3[1:] + op.E4M3[:-1]) / 2)[
        torch.randint(0, len(op.E4M3) - 1, (n // 2, 1, size), generator=g)].float()
    x[:n // 2] = half * scale
    x[:n // 2, :, 0] = (L * scale)[..., 0]
    x = x.to(TORCH[dt])
    x[7] = 0                                                                  # nothing to scale
    x[8] = torch.finfo(TORCH[dt]).tiny * 0.25                                 # below the normal numbers
    x[9] = torch.finfo(TORCH[dt]).max
    x[10, 0, 3] = float("inf")
    x[11, 0, 4] = float("nan")
    x[12, 0, 5] = -float("inf")
    x[13] = 0
    x[13, 0, 63] = -1e-4
    x[14] = -x[14].abs()
    c = empty_cache(n, 1, 1, size, kind)
    slots = torch.arange(n).cuda()
    nt.cache_write(x.cuda(), (-x).cuda(), slots, *c)
    torch.cuda.synchronize()
    for t, cache, s in ((x, c[0], c[2]), (-x, c[1], c[3])):
        code, scale = op.quantise(f64(t), kind, dt)
        assert np.array_equal(f64(s)[:, 0], scale, equal_nan=True)
        assert np.array_equal(f64(cache)[:, 0], code)
    k, v = torch.empty_like(x).cuda(), torch.empty_like(x).cuda()
    nt.cache_read(c[0], c[1], slots, k, v, c[2], c[3])
    assert k[10:13].isnan().all() and v[10:13].isnan().all() and torch.isfinite(k[:10]).all() and torch.isfinite(k[13:]).all()
    assert (k[7] == 0).all()


def test_slots_of_no_cache_are_passed_over():
    c = empty_cache(2, 4, 1, 64, "f16", fill=0x11)
    was = raw(c[0])
    k = normal((5, 1, 64), "f16", 1).cuda()
    nt.cache_write(k, k, torch.tensor([-1, 8, 3, 2 ** 40, -2 ** 63], device="cuda"), *c[:2])
    assert torch.equal(raw(c[0])[0, 3], raw(k[2]))
    assert torch.equal(raw(c[0]).index_put((torch.tensor([0]), torch.tensor([3])), was[0, 3][None]), was)


# -------------------------------------------------------------------------------------------------- attention
class Batch:
    """Sequences of given (new, length) in a cache of random pages; what no sequence holds is NaN in 16-bit caches and in scales."""

    def __init__(self, seqs, q_heads, heads, size, page, dt="f16", kind="same", layout="dense", seed=0, poison=True, before=0, behind=0):
        kind = dt if kind == "same" else kind
        self.dt, self.kind, self.page = dt, kind, page
        new, self.lengths = [s[0] for s in seqs], [s[1] for s in seqs]
        self.starts = [before + sum(new[:i]) for i in range(len(new) + 1)]
        need = [-(-max(0, n) // page) for n in self.lengths]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
        self.table = np.full((len(seqs), max(need + [1]) + 1), -1, np.int64)
        fill = 0xff if poison else 0
        self.c = empty_cache(pages, page, heads, size, kind, layout, fill)
        if poison and kind == "i8":
            self.c[0].fill_(93)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
            length = max(0, self.lengths[b])
            if not length:
                continue
            slots = torch.tensor([int(self.table[b, j // page]) * page + j % page for j in range(length)]).cuda()
            nt.cache_write(normal((length, heads, size), dt, seed + 10 * b + 1).cuda(), normal((length, heads, size), dt, seed + 10 * b + 2).cuda(), slots, *self.c)
        self.q = normal((self.starts[-1] + behind, q_heads, size), dt, seed + 5).cuda()

    def values(self):
        k, v = (f64(t) if s is None else f64(t) * f64(s)[..., None] for t, s in zip(self.c[:2], self.c[2:]))
        return k, v

    def run(self, q=None, out=None, **more):
        q = self.q if q is None else q
        out = torch.full(q.shape, -5.0, dtype=q.dtype, device="cuda") if out is None else out
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
        return nt.sdpa_paged(q, self.c[0], self.c[1], i32(self.table), i32(self.starts), i32(self.lengths), out, self.c[2], self.c[3], **more)

    def check(self, got, what="", q=None, scale=None, causal=True, window=0):
        q = self.q if q is None else q
        k, v = self.values()
        ref, A, peak = op.attend(f64(q), k, v, self.table, self.starts, self.lengths, scale, causal, window)
        got = f64(got)
        mine = slice(self.starts[0], self.starts[-1])
        assert np.array_equal(np.isnan(got[mine]), np.isnan(ref[mine])), what
        h, size, keys = torch.finfo(TORCH[self.dt]).eps / 2, q.shape[2], max(self.lengths + [1])
        top = np.abs(v[np.isfinite(v)]).max(initial=0.0)
        tol = 3.03 * h * A + 2.0 ** -24 * (size + 8) * 4 * (1 + peak) * np.sqrt(size) * A + 1e-30
        if self.dt == "f16":
            tol = tol + 2.0 ** -25 * (1 if self.kind == self.dt else 2) * min(keys, 4096) * top + 2.0 ** -25
        with np.errstate(invalid="ignore"):
            off = np.abs(got - ref) - tol
        worst = np.nanmax(off[mine], initial=-1.0)
        assert worst <= 0, f"{what}: {worst:.3g} over the bound at {np.unravel_index(np.nanargmax(off[mine]), off[mine].shape)}"
        assert (got[:self.starts[0]] == -5).all() and (got[self.starts[-1]:] == -5).all(), "rows of no sequence were written"


def attend(seqs, q_heads, heads, size, page, dt="f16", kind="same", layout="dense", seed=0, causal=True, window=0, hints=(0, 0), plan=None, **more):
    b = Batch(seqs, q_heads, heads, size, page, dt, kind, layout, seed, **more)
    got = b.run(causal=causal, window=window, max_queries=hints[0], max_length=hints[1])
    torch.cuda.synchronize()
    if plan is not None:
        p = nt.last_paged_plan()
        assert p.rows == plan[0] and plan[1] in (None, p.shares > 1), (p.rows, p.shares)
    b.check(got, causal=causal, window=window)
    return b


KINDS = [("f16", "same"), ("bf16", "same"), ("f16", "e4m3"), ("bf16", "e4m3"), ("f16", "i8"), ("bf16", "i8")]


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("q_heads,heads,size,page,layout", [(1, 1, 64, 16, "dense"), (8, 2, 128, 16, "heads first"), (6, 6, 80, 24, "dense"), (5, 1, 256, 7, "heads first"),
                                                            (4, 2, 8, 1, "dense"), (20, 1, 136, 32, "dense"), (20, 1, 120, 16, "heads first")])
def test_single_tokens(dt, kind, q_heads, heads, size, page, layout):
    """Lengths around a tile's, a page's and a share's end."""
    rows = 16 if q_heads // heads <= 16 else 32 if size <= 128 else 128
    attend([(1, n) for n in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 300)], q_heads, heads, size, page, dt, kind, layout, hints=(1, 0), plan=(rows, None))


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("q_heads,heads,size,page,layout", [(2, 2, 64, 16, "dense"), (8, 2, 128, 16, "heads first"), (3, 1, 80, 24, "dense"), (4, 2, 256, 9, "dense"), (5, 1, 40, 3, "heads first")])
def test_chunks(dt, kind, q_heads, heads, size, page, layout):
    attend([(1, 1), (70, 70), (33, 200), (1, 140), (129, 130), (0, 50), (64, 64), (40, 333)], q_heads, heads, size, page, dt, kind, layout, seed=3, plan=(128, False))


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("size", [64, 128, 256])
@pytest.mark.parametrize("layout", ["padded", "dense"])
def test_pages_of_whole_groups_of_keys(dt, kind, size, layout):
    """Whole rows, 32 keys to a page: rows at multiples of 16 bytes, and rows that begin anywhere."""
    attend([(70, 150), (1, 97), (33, 33), (130, 131)], 2, 2, size, 32, dt, kind, layout, seed=7, plan=(128, None))
    attend([(1, 150), (2, 97), (1, 1)], 2, 2, size, 32, dt, kind, layout, seed=8, hints=(2, 0), plan=(16, None))


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("size,page", [(8, 8), (40, 24), (48, 16), (72, 4), (80, 24), (96, 12), (112, 8), (136, 2), (192, 4), (248, 6), (128, 4), (256, 2), (64, 8), (64, 24), (128, 1)])
def test_sizes_between_and_pages_of_few_keys(dt, kind, size, page):
    """Chunks, with head sizes below the next built one and pages that hold a few of the rows that are fetched together, or none."""
    seqs = [(70, 150), (1, 97), (33, 33), (130, 131)]
    b = attend(seqs, 2, 2, size, page, dt, kind, seed=8, plan=(128, None))
    want = b.run().clone()
    b.table[0, 100 // page] = -1                                              # of the first sequence: keys that its last 50 tokens or more see
    got = b.run()
    b.check(got)
    first = 100 // page * page - 80
    assert torch.equal(got[:first], want[:first]) and torch.isnan(got[first + page:70]).all() and torch.equal(got[70:], want[70:])



@pytest.mark.parametrize("dt,kind", KINDS)
def test_shared_keys(dt, kind):
    """Long pasts and few programs: shares, their ends inside and beyond the shorter sequences."""
    attend([(1, 4000), (1, 5), (1, 1800), (1, 0)], 8, 2, 128, 16, dt, kind, hints=(1, 4000), plan=(16, True))
    attend([(9, 3000), (40, 41), (1, 2900)], 4, 2, 64, 16, dt, kind, hints=(40, 3000), plan=(128, True))
    attend([(3, 2500), (2, 900)], 8, 1, 128, 16, dt, kind, hints=(3, 2500), plan=(32, True))
    attend([(3, 2500), (2, 900)], 8, 1, 256, 16, dt, kind, hints=(3, 2500), plan=(128, True))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("q_heads,heads", [(1, 1), (3, 1), (16, 1), (17, 1), (48, 1), (130, 1), (12, 4)])
def test_shared_heads(dt, q_heads, heads):
    attend([(1, 77), (2, 130), (5, 40)], q_heads, heads, 64, 16, dt, seed=5)
    attend([(1, 77), (1, 200)], q_heads, heads, 64, 16, dt, seed=6, hints=(1, 200))


@pytest.mark.parametrize("kind", ["same", "e4m3"])
@pytest.mark.parametrize("window", [1, 2, 31, 64, 100, 1000])
def test_windows(kind, window):
    attend([(1, 500), (1, 30), (2, 65)], 4, 2, 64, 16, "f16", kind, window=window, hints=(2, 0))
    attend([(100, 500), (1, 30), (65, 65)], 4, 2, 64, 16, "f16", kind, window=window)
    attend([(1, 3000), (4, 2800)], 4, 2, 128, 16, "bf16", kind, window=window * 3, hints=(4, 3000))
    attend([(5, 300)], 4, 2, 64, 16, "f16", kind, window=window, causal=False)


@pytest.mark.parametrize("kind", ["same", "i8"])
def test_every_token_sees_the_whole_sequence(kind):
    attend([(1, 500), (4, 30)], 4, 2, 64, 16, "f16", kind, causal=False, hints=(4, 0))
    attend([(100, 500), (1, 30), (65, 65)], 4, 2, 128, 16, "bf16", kind, causal=False)


@pytest.mark.parametrize("kind", ["same", "e4m3"])
@pytest.mark.parametrize("hints", [(4, 0), (0, 0)])
def test_tokens_that_see_nothing(kind, hints):
    """Lengths of zero, negative ones, and fewer positions than new tokens; rows before and behind the sequences."""
    b = attend([(2, 0), (4, 1), (3, -7), (1, 9), (4, 4), (0, 0)], 4, 2, 64, 16, "bf16", kind, hints=hints, before=3, behind=5)
    got = b.run()
    assert (got[3:5] == 0).all() and (got[5:8] == 0).all() and (got[8] != 0).any() and (got[9:12] == 0).all()
    if hints[0] == 0:
        attend([(200, 20), (60, 0), (128, 127)], 4, 2, 64, 16, "f16", kind, before=1, behind=1)


@pytest.mark.parametrize("kind", ["same", "e4m3"])
@pytest.mark.parametrize("seqs,hints", [([(1, 70), (2, 33)], (2, 0)), ([(70, 150), (3, 40)], (0, 0)), ([(1, 3000)], (1, 3000))])
def test_pages_that_the_cache_does_not_have(kind, seqs, hints):
    """Seen: NaN.  Hidden by the mask: as good as any."""
    for id in (-1, 1 << 30, -2 ** 31):
        b = Batch(seqs, 4, 2, 64, 16, "f16", kind)
        b.table[0, 1] = id
        got = b.run(max_queries=hints[0], max_length=hints[1])
        b.check(got)
        assert torch.isnan(got[b.starts[1] - 1]).all()
        got = b.run(window=5, max_queries=hints[0], max_length=hints[1])
        b.check(got, window=5)
        assert torch.isfinite(got[b.starts[1] - 1]).all()
    b = Batch(seqs, 4, 2, 64, 16, "f16", kind)
    b.lengths[0] += 16 * b.table.shape[1]                                     # positions past the table's end
    got = b.run(max_queries=hints[0], max_length=hints[1])
    b.check(got)
    assert torch.isnan(got[b.starts[1] - 1]).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("size", [64, 128, 256])
def test_later_tokens_that_are_not_finite(dt, bad, size):
    """A value or key of a token that only the tokens behind it see changes nothing for those before it."""
    for seqs, hints, at in (([(4, 40), (2, 7)], (4, 0), 38), ([(100, 130), (1, 5)], (0, 0), 90), ([(3, 2000)], (3, 2000), 1998)):
        b = Batch(seqs, 4, 2, size, 16, dt, seed=9)
        want = b.run(max_queries=hints[0], max_length=hints[1]).clone()
        first = at - (seqs[0][1] - seqs[0][0])                               # the first row that sees position `at`
        page, place = int(b.table[0, at // 16]), at % 16
        was = b.c[1][page, place, 1, 3].clone()
        b.c[1][page, place, 1, 3] = bad
        got = b.run(max_queries=hints[0], max_length=hints[1])
        hit = torch.zeros_like(got, dtype=torch.bool)
        hit[first:seqs[0][0], 2:, 3] = True
        assert torch.equal(got[~hit], want[~hit])
        assert not torch.isfinite(got[hit]).any() and (torch.isnan(got[hit]).all() if bad != bad else (got[hit] == bad).all())
        b.c[1][page, place, 1, 3] = was
        if bad != -float("inf"):
            b.c[0][page, place, 1, 3] = bad
            got = b.run(max_queries=hints[0], max_length=hints[1])
            assert torch.equal(got[:first], want[:first]) and torch.equal(got[seqs[0][0]:], want[seqs[0][0]:]) and torch.equal(got[:, :2], want[:, :2])


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_scores_without_limits(dt):
    """Keys whose scores are minus infinity weigh nothing; a row with nothing else gets zeros; huge scores do not overflow."""
    for seqs, hints in (([(1, 50)], (1, 0)), ([(60, 90)], (0, 0))):
        b = Batch(seqs, 2, 2, 64, 16, dt)
        want = b.run(max_queries=hints[0])
        b.q.fill_(1.0)
        b.c[0][int(b.table[0, 0]), 3] = -float("inf")
        got = b.run(max_queries=hints[0])
        b.check(got)
        for j in range(seqs[0][1]):
            b.c[0][int(b.table[0, j // 16]), j % 16] = -float("inf")
        assert (b.run(max_queries=hints[0]) == 0).all()
        b = Batch(seqs, 2, 2, 64, 16, dt)
        q = (b.q.float() * 30).to(b.q.dtype)
        b.check(b.run(q=q, max_queries=hints[0]), q=q)
        b.check(b.run(max_queries=hints[0], scale=-0.3), scale=-0.3)
        assert torch.isfinite(want).all()


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("size_of_v", [1e-3, 3e4])
def test_values_of_any_size(kind, size_of_v):
    """fp16 weights times scales neither vanish nor overflow."""
    for seqs, hints in (([(1, 200), (1, 3)], (1, 0)), ([(60, 300)], (0, 0))):
        b = Batch(seqs, 4, 2, 64, 16, "f16", kind)
        b.c[3].mul_(size_of_v / 4)
        b.check(b.run(max_queries=hints[0]), f"{size_of_v}")
        # ... nor where one key's are far larger than those before it
        for j in range(0, seqs[0][1], 50):
            b.c[3][int(b.table[0, j // 16]), j % 16] *= 2.0 ** -20
        b.check(b.run(max_queries=hints[0]), f"{size_of_v}, mixed")


def test_a_table_without_entries():
    b = Batch([(1, 0), (2, 0)], 4, 2, 64, 16, "f16")
    b.table = np.zeros((2, 0), np.int64)
    for hints in (0, 2):
        assert (b.run(max_queries=hints) == 0).all()
    b.lengths = [1, 0]
    for hints in (0, 2):
        got = b.run(max_queries=hints)
        assert torch.isnan(got[0]).all() and (got[1:] == 0).all()


@pytest.mark.parametrize("dt,kind", [("f16", "i8"), ("f16", "e4m3"), ("bf16", "e4m3")])
def test_scales_of_later_tokens(dt, kind):
    """The scale of a key or value that a token does not see has no part in its result, however large or small or not a number."""
    for seqs, hints, at in (([(4, 40), (2, 7)], (4, 0), 38), ([(100, 130), (1, 5)], (0, 0), 90)):
        b = Batch(seqs, 4, 2, 64, 16, dt, kind, seed=9)
        want = b.run(max_queries=hints[0]).clone()
        first = at - (seqs[0][1] - seqs[0][0])
        for scales in (b.c[2], b.c[3]):
            for value in (2.0 ** 30, 2.0 ** -30, float("nan"), float("inf")):
                was = scales[int(b.table[0, at // 16]), at % 16].clone()
                scales[int(b.table[0, at // 16]), at % 16] = value
                got = b.run(max_queries=hints[0])
                assert torch.equal(got[:first], want[:first]) and torch.equal(got[seqs[0][0]:], want[seqs[0][0]:])
                scales[int(b.table[0, at // 16]), at % 16] = was


def test_strided_queries_and_outputs():
    b = Batch([(1, 50), (30, 60)], 4, 2, 80, 16, "bf16")
    wide = torch.full((4, 31, 93), -9.0, dtype=torch.bfloat16, device="cuda")
    q = wide[:, :, 5:85].permute(1, 0, 2)
    q.copy_(b.q)
    buf = torch.full((31, 4, 91), -5.0, dtype=torch.bfloat16, device="cuda")
    for hints in (0, 2):
        b.check(b.run(q=q, out=buf[..., 3:83], max_queries=hints))
        assert (buf[..., :3] == -5).all() and (buf[..., 83:] == -5).all()


def test_bounds_that_are_too_low_cost_time_only():
    b = Batch([(1, 50), (70, 300), (9, 9)], 4, 2, 64, 16, "f16")
    for hints in ((1, 1), (3, 40), (8, 0), (64, 100)):
        b.check(b.run(max_queries=hints[0], max_length=hints[1]), str(hints))


def test_offsets_beyond_32_bits():
    """Pages that lie more than 2^32 bytes apart: a cache in a buffer of 5 GB."""
    size, heads, page = 64, 2, 16
    buf = torch.zeros(5 << 30, dtype=torch.uint8, device="cuda")
    for dt, kind in (("f16", "same"), ("bf16", "e4m3")):
        b = Batch([(1, 40), (20, 45)], 4, heads, size, page, dt, kind, poison=False)
        pages = b.c[0].shape[0]
        far = []
        for t in b.c[:2]:
            es, per = t.element_size(), page * heads * size
            step = ((5 << 30) // es - per * 4) // pages // 64 * 64
            w = buf.view(t.dtype).as_strided((pages, page, heads, size), (step, heads * size, size, 1), 64 * len(far) * heads * page)
            w.view(torch.uint8 if es == 1 else t.dtype).copy_(t.view(torch.uint8 if es == 1 else t.dtype))
            far.append(w)
        want = [b.run(max_queries=m) for m in (2, 0)]
        b.c = (far[0], far[1], b.c[2], b.c[3])
        got = [b.run(max_queries=m) for m in (2, 0)]
        assert all(torch.equal(g, w) for g, w in zip(got, want))
        k, v = normal((3, heads, size), dt, 1).cuda(), normal((3, heads, size), dt, 2).cuda()
        slots = torch.tensor([0, page * pages - 1, page * (pages // 2)], device="cuda")
        nt.cache_write(k, v, slots, *b.c)
        back = torch.empty_like(k), torch.empty_like(v)
        nt.cache_read(b.c[0], b.c[1], slots, back[0], back[1], b.c[2], b.c[3])
        assert (back[0].float() - k.float()).abs().max() <= (0 if kind == "same" else 0.2)


class Tagged(torch.Tensor):
    """A tensor subclass: marshalled by the binding itself."""


@pytest.mark.parametrize("kind", ["same", "i8"])
def test_every_way_gives_the_same_bits(kind):
    b = Batch([(1, 3000), (2, 40)], 4, 2, 64, 16, "f16", kind)
    want = b.run(max_queries=2, max_length=3000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [b.run(q=b.q.as_subclass(Tagged), max_queries=2, max_length=3000), b.run(max_queries=2, max_length=3000, stream=torch.cuda.current_stream())]
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.empty_like(b.q)
    call = nt.prepare(nt.sdpa_paged, b.q, b.c[0], b.c[1], i32(b.table), i32(b.starts), i32(b.lengths), out, b.c[2], b.c[3], max_queries=2, max_length=3000)
    call()
    got.append(out)
    with torch.cuda.stream(side):
        got.append(b.run(max_queries=2, max_length=3000))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    k = normal((5, 2, 64), "f16", 4).cuda()
    slots = torch.arange(5, device="cuda")
    made = []
    for f in (lambda t: t, lambda t: t.as_subclass(Tagged)):
        c = empty_cache(1, 8, 2, 64, b.kind)
        nt.cache_write(f(k), k, slots, *c)
        r = torch.empty_like(k), torch.empty_like(k)
        nt.cache_read(c[0], c[1], slots, f(r[0]), r[1], c[2], c[3])
        made.append([raw(t) for t in (*[x for x in c if x is not None], *r)])
    assert all(torch.equal(x, y) for x, y in zip(*made))


def test_errors_of_arguments():
    b = Batch([(1, 30)], 4, 2, 64, 16, "f16", "e4m3")
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    a = [b.q, b.c[0], b.c[1], i32(b.table), i32(b.starts), i32(b.lengths), torch.empty_like(b.q), b.c[2], b.c[3]]

    def refused(error, **over):
        args = [over.get(n, x) for n, x in zip(("q", "k", "v", "table", "starts", "lengths", "out", "ks", "vs"), a)]
        with pytest.raises(error):
            nt.sdpa_paged(*args)
    refused(ValueError, table=a[3].long())
    refused(ValueError, starts=a[4].long())
    refused(ValueError, starts=a[4][:1])
    refused(ValueError, lengths=i32([1, 2]))
    refused(ValueError, lengths=i32([1, 2, 3, 4])[::2])
    refused(ValueError, out=a[6].float())
    refused(ValueError, v=a[2].view(torch.int8))
    refused(ValueError, ks=None)
    refused(ValueError, ks=a[7].half(), vs=a[8].half())
    refused(nt.NtError, ks=None, vs=None)
    refused(nt.NtError, q=a[0][..., :56], out=a[6][..., :56])
    k = normal((2, 2, 64), "f16", 1).cuda()
    for slots in (torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int64)):
        with pytest.raises(ValueError):
            nt.cache_write(k, k, slots, *b.c)
    with pytest.raises(ValueError):
        nt.cache_write(k, k.bfloat16(), torch.zeros(2, dtype=torch.int64, device="cuda"), *b.c)
    nt.sdpa_paged(*a)


@pytest.mark.parametrize("seqs,hints", [([(1, 4000), (1, 60)], (1, 4000)), ([(40, 2000), (1, 60)], (40, 2000)), ([(1, 100)], (1, 100))])
def test_captured_into_a_graph(seqs, hints):
    """Replays, on changing inputs, with eager calls of the same kind between them."""
    b = Batch(seqs, 4, 2, 64, 16, "f16", "e4m3")
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    table, starts, lengths, out = i32(b.table), i32(b.starts), i32(b.lengths), torch.empty_like(b.q)
    k, v, slot = normal((1, 2, 64), "f16", 3).cuda(), normal((1, 2, 64), "f16", 4).cuda(), torch.tensor([int(b.table[0, 0]) * 16], device="cuda")

    def step(o):
        nt.cache_write(k, v, slot, *b.c)
        nt.sdpa_paged(b.q, b.c[0], b.c[1], table, starts, lengths, o, b.c[2], b.c[3], max_queries=hints[0], max_length=hints[1])
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for i in range(4):
        k.copy_(normal((1, 2, 64), "f16", 20 + i))
        b.q.copy_(normal(b.q.shape, "f16", 30 + i))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(out)
        step(want)
        assert torch.equal(out, want)
        step(want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_two_streams():
    """Shares of calls on two streams meet in the workspace."""
    bs = [Batch([(1, 3500), (1, 2000)], 4, 2, 64, 16, "f16", seed=s) for s in (1, 2)]
    want = [b.run(max_queries=1, max_length=3500).clone() for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, (b, s) in enumerate(zip(bs, streams)):
            with torch.cuda.stream(s):
                got[i].append(b.run(max_queries=1, max_length=3500))
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for g, w in zip(got, want) for x in g)
