"""GPU parity of drafted tokens over a paged cache (cache_fit, tree_masks, sdpa_paged_tree, verify_tree, cache_compact) against the plain definitions.

All but the attention are exact: whole numbers, and elements that are moved as they are.

Attention.  The result's rounding: h |O| with h = eps / 2 of its type (fp16: 2^-25 at least).  A score is an fp32 sum of `size` products, some eight more roundings follow
until its exponential: off by 2^-24 (size + 8) S at most, with S the largest of scale * sum |q| |k| over the keys that the row sees; that is the relative error
of a weight, and twice that of the quotient.  Sums over n keys, and of the shares, in fp32: 2^-24 (n + 64).  A weight multiplies V as two 16-bit numbers: off by 2^-16 of it in bf16 (over codes in either type), 2^-22
in fp16, there 2^-24 of a weight of 1 besides, for each key (the rest is that at least, and rounded to multiples of it; no row's reference is above its largest weight).
All of these but the first and last are relative to A = sum_j p_j |V_j|, the last to the largest |V|."""
import numpy as np
import pytest
import torch

import paper_2507_11978_amd as nt
from oracle import tree as ot
from test_gpu_paged import KINDS, TORCH, Tagged, empty_cache, f64, normal, raw

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def i64(x):
    return torch.tensor(np.asarray(x), dtype=torch.int64, device="cuda")


def every_byte(t):
    return t.contiguous().view(torch.uint8).cpu()


def random_tree(n, g):
    return [-1 if i == 0 else int(g.integers(max(0, i - 1 - int(g.integers(1, 9))), i)) for i in range(n)]


class Trees:
    """Sequences of (new tokens, length with them) in a cache of random pages; what no sequence holds is NaN in 16-bit caches and in scales."""

    def __init__(self, seqs, q_heads, heads, size, page, dt="f16", kind="same", layout="dense", seed=0, before=0, behind=0, poison=True, words=None, bits="tree", window=0):
        kind = dt if kind == "same" else kind
        self.dt, self.kind, self.page, self.window = dt, kind, page, window
        new, self.lengths = [s[0] for s in seqs], [s[1] for s in seqs]
        self.starts = [before + sum(new[:i]) for i in range(len(new) + 1)]
        need = [-(-max(0, n) // page) for n in self.lengths]
        pages = sum(need) + 3
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
        self.table = np.full((len(seqs), max(need + [1]) + 1), -1, np.int64)
        self.c = empty_cache(pages, page, heads, size, kind, layout, 0xff if poison else 0)
        if poison and kind == "i8":
            self.c[0].fill_(93)
        at, slots = 0, []
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
            slots += [int(self.table[b, j // page]) * page + j % page for j in range(max(0, self.lengths[b]))]
        if slots:
            k, v = (normal((len(slots), heads, size), dt, seed + i).cuda() for i in (1, 2))
            nt.cache_write(k, v, i64(slots), *self.c)
        T = self.starts[-1] + behind
        self.q = normal((T, q_heads, size), dt, seed + 5).cuda()
        g = np.random.default_rng(seed)
        words = -(-max(new + [1]) // 64) if words is None else words
        self.mask, self.depths = np.zeros((T, words), np.int64), np.zeros(T, np.int64)
        for b, n in enumerate(new):
            seen, depths = ot.ancestors(random_tree(n, g), window)
            self.mask[self.starts[b]:self.starts[b + 1]] = ot.masks(seen, words)
            self.depths[self.starts[b]:self.starts[b + 1]] = depths
        if bits == "any":                                                     # no tree: whoever sees whomever, some no one
            self.mask = g.integers(-2 ** 63, 2 ** 63, self.mask.shape)
            self.mask[g.random(T) < 0.2] = 0

    def values(self):
        return [f64(t) if s is None else f64(t) * f64(s)[..., None] for t, s in zip(self.c[:2], self.c[2:])]

    def args(self, q=None, out=None, masks=None):
        q = self.q if q is None else q
        out = torch.full(q.shape, -5.0, dtype=q.dtype, device="cuda") if out is None else out
        return (q, self.c[0], self.c[1], i32(self.table), i32(self.starts), i32(self.lengths), i64(self.mask) if masks is None else masks, out, self.c[2], self.c[3])

    def run(self, q=None, out=None, masks=None, **more):
        if self.window:
            more.update(window=self.window, depths=i32(self.depths))
        return nt.sdpa_paged_tree(*self.args(q, out, masks), **more)

    def check(self, got, what="", q=None, scale=None):
        q = self.q if q is None else q
        k, v = self.values()
        ref, A, S = ot.attend(f64(q), k, v, self.table, self.starts, self.lengths, self.mask, self.depths, self.window, scale)
        got = f64(got)
        mine = slice(self.starts[0], self.starts[-1])
        assert np.array_equal(np.isnan(got[mine]), np.isnan(ref[mine])), what
        n, h = min(max(self.lengths + [1]), 1 << 20), torch.finfo(TORCH[self.dt]).eps / 2
        tol = 1.01 * h * np.abs(ref) + A * (2.0 ** -24 * (2 * (q.shape[2] + 8) * S + n + 64) + 1.01 * 2.0 ** -16) + 1e-30
        if self.dt == "f16":
            tol = tol + 2.0 ** -25
            if self.kind == "f16":
                tol = tol + 2.0 ** -24 * n * np.abs(v[np.isfinite(v)]).max(initial=0.0)
        with np.errstate(invalid="ignore"):
            off = np.abs(got - ref) - tol
            off[np.isinf(ref) & (got == ref)] = -1.0
        worst = np.nanmax(off[mine], initial=-1.0)
        assert worst <= 0, f"{what}: {worst:.3g} over the bound at {np.unravel_index(np.nanargmax(off[mine]), off[mine].shape)}"
        assert (got[:self.starts[0]] == -5).all() and (got[self.starts[-1]:] == -5).all(), "rows of no sequence were written"


def attend(seqs, q_heads, heads, size, page, dt="f16", kind="same", layout="dense", seed=0, hints=(0, 0), rows=None, **more):
    b = Trees(seqs, q_heads, heads, size, page, dt, kind, layout, seed, **more)
    got = b.run(max_queries=hints[0], max_length=hints[1])
    torch.cuda.synchronize()
    if rows is not None:
        assert nt.last_paged_plan().rows == rows
    b.check(got)
    return b


MANY = [(1, 1), (8, 8), (16, 200), (0, 50), (7, 70), (33, 300), (64, 65), (64, 64), (5, 129)]


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("q_heads,heads,size,page,layout", [(1, 1, 64, 16, "dense"), (8, 2, 128, 16, "heads first"), (6, 6, 80, 24, "dense"), (3, 1, 256, 7, "heads first"),
                                                            (4, 2, 8, 1, "dense"), (5, 5, 136, 32, "padded"), (4, 1, 120, 16, "padded")])
def test_trees(dt, kind, q_heads, heads, size, page, layout):
    """Lengths around a block's and a page's end, no past, no new tokens."""
    attend(MANY, q_heads, heads, size, page, dt, kind, layout, before=2, behind=3, hints=(64, 300), rows=64 if 64 * q_heads // heads <= 64 and size <= 128 else 128)


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("size", [64, 128, 256])
def test_masks_of_any_bits(dt, kind, size):
    """Tokens that see others than their ancestors, or no new token at all, with a past and without one; more words than new tokens, and fewer."""
    attend([(70, 70), (16, 300), (130, 140), (3, 3), (64, 200)], 2, 2, size, 16, dt, kind, seed=3, bits="any", words=3)
    attend([(5, 70), (16, 300), (3, 3)], 4, 2, size, 16, dt, kind, seed=4, bits="any", words=2, hints=(16, 0))
    attend([(100, 170), (16, 16)], 2, 1, size, 32, dt, kind, seed=5, bits="any", words=1)


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("q_heads,heads", [(1, 1), (3, 1), (16, 1), (48, 3), (12, 4), (130, 1)])
def test_shared_heads(dt, kind, q_heads, heads):
    attend([(9, 77), (2, 130), (5, 40)], q_heads, heads, 64, 16, dt, kind, seed=5)
    attend([(2, 77), (1, 200), (1, 3)], q_heads, heads, 128, 16, dt, kind, seed=6, hints=(2, 200))


@pytest.mark.parametrize("dt,kind", [("f16", "same"), ("bf16", "i8")])
def test_sequences_of_every_age(dt, kind):
    """Runs of blocks that end inside a sequence, at its beginning and its end, and hold many."""
    g = np.random.default_rng(4)
    for seed, (B, longest) in enumerate([(40, 900), (100, 200), (7, 5000), (3, 3000), (1, 6000), (300, 90)]):
        lengths = [int(n) for n in np.exp(g.uniform(0, np.log(longest), B))]
        lengths[0] = longest
        attend([(int(g.integers(0, min(n, 12) + 1)), n) for n in lengths], 2, 2, 64, 16, dt, kind, seed=seed, hints=(12, 0))
    attend([(20, 1000), (20, 1), (33, 2000)], 8, 2, 128, 16, dt, kind, seed=9)
    attend([(20, 1000), (20, 21), (33, 2000)], 2, 2, 256, 16, dt, kind, seed=9)


def test_more_sequences_than_are_dealt_out():
    attend([(i % 3, 2 + i % 70) for i in range(1100)], 2, 1, 64, 16, "bf16", hints=(2, 0))
    attend([(1, 30)] * 1024, 1, 1, 64, 16, "f16", hints=(1, 0))
    attend([(1, 30)] * 1023 + [(3, 300)], 1, 1, 64, 16, "f16")


@pytest.mark.parametrize("kind", ["same", "e4m3"])
@pytest.mark.parametrize("window", [1, 2, 5, 31, 64, 100, 1000])
def test_windows(kind, window):
    attend([(40, 500), (9, 30), (20, 20), (1, 65)], 4, 2, 64, 16, "f16", kind, window=window)
    attend([(12, 3000), (4, 2800)], 4, 2, 128, 16, "bf16", kind, window=window * 3, hints=(12, 3000))
    b = attend([(12, 300)], 4, 2, 64, 16, "f16", kind, window=window, bits="any")
    want = b.run().clone()
    b.depths = np.where(b.depths == 0, -7, b.depths)                          # (0 to n - 1 is what they are taken as)
    assert torch.equal(b.run(), want)


@pytest.mark.parametrize("kind", ["same", "e4m3"])
@pytest.mark.parametrize("hints", [(4, 0), (0, 0), (1, 1)])
def test_tokens_that_see_nothing(kind, hints):
    """Lengths of zero, negative ones, fewer positions than new tokens; masks without a bit; rows before and behind the sequences."""
    b = Trees([(2, 0), (4, 1), (3, -7), (1, 9), (4, 4), (0, 0), (3, 3)], 4, 2, 64, 16, "bf16", kind, before=3, behind=5)
    b.mask[b.starts[6]:] = 0
    got = b.run(max_queries=hints[0], max_length=hints[1])
    b.check(got)
    assert (got[3:5] == 0).all() and (got[9:12] == 0).all() and (got[12] != 0).any() and (got[b.starts[6]:b.starts[7]] == 0).all()


@pytest.mark.parametrize("kind", ["same", "e4m3"])
@pytest.mark.parametrize("seqs,hints", [([(9, 70), (2, 33)], (9, 0)), ([(70, 150), (3, 40)], (0, 0)), ([(4, 3000)], (4, 3000))])
def test_pages_that_the_cache_does_not_have(kind, seqs, hints):
    """Seen: NaN.  Hidden by mask or window: as good as any."""
    for id in (-1, 1 << 30, -2 ** 31):
        b = Trees(seqs, 4, 2, 64, 16, "f16", kind)
        b.table[0, 1] = id
        got = b.run(max_queries=hints[0], max_length=hints[1])
        b.check(got)
        assert torch.isnan(got[:seqs[0][0]]).all()
        b = Trees(seqs, 4, 2, 64, 16, "f16", kind, window=5)
        b.table[0, 1] = id
        got = b.run(max_queries=hints[0], max_length=hints[1])
        b.check(got)
        b = Trees(seqs, 4, 2, 64, 16, "f16", kind)                            # a page of new tokens: those that see one of it
        b.table[0, (seqs[0][1] - 1) // 16] = id
        got = b.run(max_queries=hints[0], max_length=hints[1])
        b.check(got)
    for window in (0, 1, 3):
        b = Trees(seqs, 4, 2, 64, 16, "f16", kind, window=window)
        b.lengths[0] += 16 * b.table.shape[1]                                 # positions past the table's end
        b.mask[0] = 0
        got = b.run(max_queries=hints[0], max_length=hints[1])
        b.check(got)
        assert torch.isnan(got[1:seqs[0][0]]).all() and (window != 1 or (got[0] == 0).all())
        b = Trees(seqs, 4, 2, 64, 16, "f16", kind, window=window)
        b.lengths[0] += 3                                                     # ... of some
        b.table = b.table[:, :-(-seqs[0][1] // 16)]
        b.check(b.run(max_queries=hints[0], max_length=hints[1]))


@pytest.mark.parametrize("kind", ["same", "i8"])
@pytest.mark.parametrize("window", [0, 4])
def test_lengths_that_no_table_reaches(kind, window):
    """Lengths up to 2^31 - 1: NaN for those that see anything, and no walk of 2^31 keys."""
    for length in (2 ** 31 - 1, 2 ** 31 - 4097, 2 ** 30):
        b = Trees([(9, 200), (70, 100)], 2, 2, 64, 16, "f16", kind, window=window)
        want = b.run().clone()
        b.lengths[0] = length
        b.mask[1] = 0
        got = b.run()
        assert torch.isnan(got[2:9]).all() and torch.isnan(got[0]).all() and torch.equal(got[9:], want[9:])
        assert torch.isnan(got[1]).all() or (window and (got[1] == 0).all())


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("size", [64, 128, 256])
def test_others_that_are_not_finite(dt, bad, size):
    """A value or key of a token that only its descendants see changes nothing for the others."""
    for seqs, hints, at in (([(9, 40), (2, 7)], (9, 0), 3), ([(100, 130), (1, 5)], (0, 0), 60), ([(5, 2000)], (5, 2000), 1)):
        b = Trees(seqs, 4, 2, size, 16, dt, seed=9)
        want = b.run(max_queries=hints[0], max_length=hints[1]).clone()
        n = seqs[0][0]
        sees = torch.tensor([(int(b.mask.view(np.uint64)[i, at // 64]) >> (at % 64)) & 1 == 1 for i in range(n)])
        assert 0 < sees.sum() < n
        p = seqs[0][1] - n + at
        page, place = int(b.table[0, p // 16]), p % 16
        was = b.c[1][page, place, 1, 3].clone()
        b.c[1][page, place, 1, 3] = bad
        got = b.run(max_queries=hints[0], max_length=hints[1])
        hit = torch.zeros_like(got, dtype=torch.bool)
        hit[:n, 2:, 3] = sees[:, None].cuda()
        assert torch.equal(got[~hit], want[~hit])
        assert torch.isnan(got[hit]).all() if bad != bad else (got[hit] == bad).all()
        b.c[1][page, place, 1, 3] = was
        if bad != -float("inf"):
            b.c[0][page, place, 1, 3] = bad
            got = b.run(max_queries=hints[0], max_length=hints[1])
            hit = torch.zeros_like(got, dtype=torch.bool)
            hit[:n, 2:] = sees[:, None, None].cuda()
            assert torch.equal(got[~hit], want[~hit])


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_values_that_all_see_and_are_not_finite(dt, bad):
    """An infinity that every row sees, in blocks without a mask, with weights of every size, stays one."""
    for size, at in ((64, 70), (128, 5), (256, 100)):
        b = Trees([(5, 400), (3, 90)], 2, 1, size, 16, dt, seed=2)
        want = b.run().clone()
        b.c[1][int(b.table[0, at // 16]), at % 16, 0, 7] = bad
        got = b.run()
        hit = torch.zeros_like(got, dtype=torch.bool)
        hit[:5, :, 7] = True
        assert torch.equal(got[~hit], want[~hit]) and (torch.isnan(got[hit]).all() if bad != bad else (got[hit] == bad).all())


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_scores_without_limits(dt):
    """Keys whose scores are minus infinity weigh nothing; a row with nothing else gets zeros; huge scores do not overflow; late keys far above the others count."""
    for seqs in ([(5, 50)], [(60, 190)], [(4, 2000)]):
        b = Trees(seqs, 2, 2, 64, 16, dt)
        b.q.fill_(1.0)
        b.c[0][int(b.table[0, 0]), 3] = -float("inf")
        b.check(b.run())
        for j in range(seqs[0][1]):
            b.c[0][int(b.table[0, j // 16]), j % 16] = -float("inf")
        assert (b.run() == 0).all()
        b = Trees(seqs, 2, 2, 64, 16, dt)
        q = (b.q.float() * 30).to(b.q.dtype)
        b.check(b.run(q=q), q=q)
        b.check(b.run(scale=-0.3), scale=-0.3)
        for late in (seqs[0][1] - seqs[0][0] - 1, seqs[0][1] - seqs[0][0]):   # the past's last, the root
            b.q[..., 0] = 8.0
            b.c[0][int(b.table[0, late // 16]), late % 16, :, 0] = 40.0
            b.check(b.run(), f"late {late}")


@pytest.mark.parametrize("dt,kind", [("f16", "i8"), ("f16", "e4m3"), ("bf16", "e4m3")])
def test_scales_of_others(dt, kind):
    """The scale of a key or value that a token does not see has no part in its result, however large or small or not a number; values of any size do not overflow."""
    for seqs, at in (([(9, 40), (2, 7)], 5), ([(100, 130), (1, 5)], 60)):
        b = Trees(seqs, 4, 2, 64, 16, dt, kind, seed=9)
        want = b.run().clone()
        n, p = seqs[0][0], seqs[0][1] - seqs[0][0] + at
        sees = torch.tensor([(int(b.mask.view(np.uint64)[i, at // 64]) >> (at % 64)) & 1 == 1 for i in range(n)] + [False] * (b.q.shape[0] - n)).cuda()
        for scales in (b.c[2], b.c[3]):
            for value in (2.0 ** 30, 2.0 ** -30, float("nan"), float("inf")):
                was = scales[int(b.table[0, p // 16]), p % 16].clone()
                scales[int(b.table[0, p // 16]), p % 16] = value
                assert torch.equal(b.run()[~sees], want[~sees])
                scales[int(b.table[0, p // 16]), p % 16] = was
        b.c[3].mul_(3e4 / 4)
        b.check(b.run())


def test_strides():
    b = Trees([(9, 50), (30, 60)], 4, 2, 80, 16, "bf16", words=2)
    wide = torch.full((4, 39, 93), -9.0, dtype=torch.bfloat16, device="cuda")
    q = wide[:, :, 5:85].permute(1, 0, 2)
    q.copy_(b.q)
    buf = torch.full((39, 4, 91), -5.0, dtype=torch.bfloat16, device="cuda")
    masks = torch.full((39, 5), -1, dtype=torch.int64, device="cuda")[:, 2:4]
    masks.copy_(i64(b.mask))
    for hints in (0, 30):
        b.check(b.run(q=q, out=buf[..., 3:83], masks=masks, max_queries=hints))
        assert (buf[..., :3] == -5).all() and (buf[..., 83:] == -5).all()


def test_bounds_that_are_too_low_cost_time_only():
    b = Trees([(3, 50), (70, 300), (9, 9), (200, 200)], 4, 2, 64, 16, "f16")
    for hints in ((1, 1), (3, 40), (8, 0), (64, 100), (0, 0)):
        b.check(b.run(max_queries=hints[0], max_length=hints[1]), str(hints))
    b = Trees([(70, 300), (2, 9)], 4, 2, 256, 16, "bf16", "e4m3")
    b.check(b.run(max_queries=1))


def test_a_table_without_entries():
    b = Trees([(1, 0), (3, 0)], 4, 2, 64, 16, "f16")
    b.table = np.zeros((2, 0), np.int64)
    assert (b.run() == 0).all()
    b.lengths = [1, 0]
    got = b.run()
    assert torch.isnan(got[0]).all() and (got[1:] == 0).all()


def test_rows_beyond_the_bound_among_sequences():
    """A tree far larger than the others', and than the bound: its rows are dealt out among the programs that share its keys."""
    b = Trees([(1, 100), (300, 900), (2, 500), (1, 3), (150, 150), (1, 700)], 4, 2, 64, 16, "bf16", words=5)
    want = b.run(max_queries=300).clone()
    b.check(want)
    for m in (1, 2, 20, 0):
        b.check(b.run(max_queries=m), str(m))


def test_offsets_beyond_32_bits():
    """Pages that lie more than 2^32 bytes apart: a cache in a buffer of 5 GB."""
    size, heads, page = 64, 2, 16
    buf = torch.zeros(5 << 30, dtype=torch.uint8, device="cuda")
    for dt, kind in (("f16", "same"), ("bf16", "e4m3")):
        b = Trees([(5, 40), (20, 45)], 4, heads, size, page, dt, kind, poison=False)
        pages, far = b.c[0].shape[0], []
        for t in b.c[:2]:
            es, per = t.element_size(), page * heads * size
            step = ((5 << 30) // es - per * 4) // pages // 64 * 64
            w = buf.view(t.dtype).as_strided((pages, page, heads, size), (step, heads * size, size, 1), 64 * len(far) * heads * page)
            w.view(torch.uint8 if es == 1 else t.dtype).copy_(t.view(torch.uint8 if es == 1 else t.dtype))
            far.append(w)
        want = b.run()
        near = [t.clone() for t in b.c if t is not None]
        near = near + [None] * (4 - len(near))
        b.c = (far[0], far[1], b.c[2], b.c[3])
        assert torch.equal(b.run(), want)
        args = i32(b.table), i32([40, 45]), i32([[0, 2, 3], [0, 4, 19]]), i32([3, 2])
        nt.cache_compact([b.c[:2] if kind == "same" else b.c], *args)
        nt.cache_compact([tuple(near[:2]) if kind == "same" else tuple(near)], *args)
        for w, t in zip(far, near[:2]):
            assert torch.equal(raw(w), raw(t))


# ------------------------------------------------------------------------------------------------------------ pages and slots
class Pool:
    """A cache's pages, kept by the oracle and on the GPU."""

    def __init__(self, B, pages, page, width, seed, strided=False):
        g = np.random.default_rng(seed)
        self.g, self.page, self.B = g, page, B
        self.table, self.held = np.full((B, width), -9, np.int64), [0] * B
        self.free, self.count = [int(x) for x in g.permutation(pages)], pages
        self.lengths = [0] * B
        t = torch.full((B, width + 7), -9, dtype=torch.int32, device="cuda")
        self.d_table = t[:, 3:3 + width] if strided else t[:, :width].contiguous()
        self.d_held, self.d_free, self.d_count = i32(self.held), i32(self.free), i32([self.count])
        self.d_starts, self.d_new = i32([-3] * (B + 1)), i32([-3] * B)

    def step(self, lengths, counts, tokens=None, alias=False):
        total = sum(max(0, c) for c in counts)
        tokens = total if tokens is None else tokens
        slots, positions = i64([-3] * tokens), i32([-3] * tokens)
        n = i32(lengths)
        new = n if alias else self.d_new
        nt.cache_fit(n, i32(counts), self.page, self.d_table, self.d_held, self.d_free, self.d_count, self.d_starts, new, slots, positions)
        starts, want, s, p, self.count = ot.fit(lengths, counts, self.page, self.table, self.held, self.free, self.count, tokens)
        self.lengths = want
        assert self.d_starts.tolist() == starts and new.tolist() == want
        assert self.d_held.tolist() == self.held and self.d_count.item() == self.count
        assert np.array_equal(self.d_table.cpu().numpy(), self.table)
        top = max(0, self.count)
        assert self.d_free.tolist()[:top] == self.free[:top]
        assert slots.tolist() == s and positions.tolist() == p


@pytest.mark.parametrize("B,page,strided", [(1, 16, False), (5, 1, True), (64, 24, False), (300, 16, True), (1024, 7, False), (1025, 16, False), (3000, 32, False)])
def test_pages_come_and_go(B, page, strided):
    g = np.random.default_rng(B)
    longest = 2000 if B < 100 else 120
    width = -(-longest // page) + 2
    p = Pool(B, B * width, page, width, B, strided)
    for step in range(5):
        over = g.random(B) < (0.3 if step else 0)
        lengths = [0 if o else n for o, n in zip(over, p.lengths)]
        room = [longest - n for n in lengths]
        counts = [int(g.integers(0, r + 1)) if o or step == 0 else min(r, int(g.integers(0, 3))) for o, r in zip(over, room)]
        p.step(lengths, counts, alias=step % 2 == 1)
        # drafts that did not stand: shorter again, pages beyond go back with the next call
        p.lengths = [max(0, n - int(g.integers(0, 2 * page))) for n in p.lengths]
    p.step([0] * B, [0] * B)
    assert p.count == B * width and sorted(p.free) == list(range(B * width))


def test_pages_that_come_back_are_taken_in_the_same_order():
    p = Pool(6, 60, 16, 10, 1)
    p.step([0] * 6, [100, 3, 50, 0, 16, 17])
    was = p.d_table.clone()
    p.step([0] * 6, [0] * 6)
    p.step([0] * 6, [100, 3, 50, 0, 16, 17])
    assert torch.equal(p.d_table, was)


def test_more_than_there_is():
    """The stack runs out, rows of the table end, and there is room for the next call when pages come back."""
    p = Pool(4, 10, 16, 6, 2)
    p.step([0] * 4, [40, 0, 90, 80])                                          # 3 + 6 + 5 pages of 10
    assert p.count == -4 and p.held == [3, 0, 6, 1]
    p.step(p.lengths, [0, 5, 0, 0])
    p.step([40, 0, 0, 0], [1, 5, 200, 3])                                     # (200 do not fit a row of 6)
    p.step([0, 0, 0, 0], [0, 0, 0, 0])
    assert p.count == 10
    p = Pool(2, 0, 16, 3, 2)
    p.step([0, 0], [5, 0])
    p = Pool(2, 5, 16, 0, 2)
    p.step([0, 0], [5, 1])


def test_slots_for_more_and_fewer_tokens():
    """Padding behind the last token; fewer slots than tokens; many tokens; counts and lengths below zero; no tokens; no sequences."""
    p = Pool(3, 2000, 16, 600, 3)
    p.step([0, 0, 0], [5, 0, 7], tokens=40)
    p.step(p.lengths, [30, 1, 2], tokens=10)
    p.step(p.lengths, [6000, 1, 2000], tokens=9000)
    p.step(p.lengths, [-5, -1, 2])
    p.step([-4, 10, 3], [0, 0, 0], tokens=5)
    p.step([0, 0, 0], [4096, 0, 0])
    p.step([0, 0, 0], [4097, 0, 0])
    starts, count = i32([7]), i32([3])
    e = i32([])
    slots, positions = i64([5, 5]), i32([5, 5])
    nt.cache_fit(e, e, 16, torch.empty((0, 4), dtype=torch.int32, device="cuda"), e, i32([1, 2, 3]), count, starts, e, slots, positions)
    assert starts.tolist() == [0] and count.tolist() == [3] and slots.tolist() == [-1, -1] and positions.tolist() == [0, 0]


# ------------------------------------------------------------------------------------------------------------ masks
def masked(trees, words, window=0, before=0, behind=0, lengths=None):
    T = before + sum(map(len, trees)) + behind
    starts = [before + sum(map(len, trees[:i])) for i in range(len(trees) + 1)]
    parents = i32([5] * before + [p for t in trees for p in t] + [5] * behind)
    wide = torch.full((T, words + 3), 77, dtype=torch.int64, device="cuda")
    depths, positions = i32([-3] * T), i32([-3] * T)
    lengths = [10 * i + len(t) for i, t in enumerate(trees)] if lengths is None else lengths
    nt.tree_masks(parents, i32(starts), wide[:, 1:1 + words], depths, i32(lengths), positions, window=window)
    want, want_d, want_p = np.full((T, words), 77), np.full(T, -3), np.full(T, -3)
    for t, s, n in zip(trees, starts, lengths):
        seen, d = ot.ancestors(t, window)
        if len(t):
            want[s:s + len(t)], want_d[s:s + len(t)] = ot.masks(seen, words), d
            want_p[s:s + len(t)] = n - len(t) + np.array(d)
    got = wide.cpu().numpy()
    assert np.array_equal(got[:, 1:1 + words], want) and (got[:, 0] == 77).all() and (got[:, 1 + words:] == 77).all()
    assert depths.tolist() == want_d.tolist() and positions.tolist() == want_p.tolist()


@pytest.mark.parametrize("window", [0, 1, 3, 64, 1000])
def test_masks(window):
    g = np.random.default_rng(window)
    masked([random_tree(n, g) for n in (1, 8, 0, 64, 65, 3, 128, 1, 200)], 4, window, 3, 2)
    masked([random_tree(n, g) for n in (8, 100)], 1, window)                  # (bits that there is no room for)
    masked([list(range(-1, 2999)), [-1] * 300, [0, -5, 1, 3, 2, 99, 5]], 47, window)        # a long chain; roots only; parents that are none
    masked([[-1, 2 ** 31 - 1, -2 ** 31, 0]], 1, window)


def test_masks_without_positions_and_without_tokens():
    m, d = torch.full((3, 1), 7, dtype=torch.int64, device="cuda"), i32([7] * 3)
    nt.tree_masks(i32([-1, 0, 0]), i32([0, 3]), m, d)
    assert m[:, 0].tolist() == [1, 3, 5] and d.tolist() == [0, 1, 1]
    nt.tree_masks(i32([-1, 0, 0]), i32([0]), m, d)
    nt.tree_masks(i32([]), i32([0, 0]), m[:0], d[:0])
    assert m[:, 0].tolist() == [1, 3, 5]


# ------------------------------------------------------------------------------------------------------------ verification
class Drafts:
    def __init__(self, trees, V, dt="f32", drafted=True, seed=0, before=0, behind=0, sure=3.0, pad=0):
        g = torch.Generator().manual_seed(seed)
        T = before + sum(map(len, trees)) + behind
        self.starts = [before + sum(map(len, trees[:i])) for i in range(len(trees) + 1)]
        x = torch.randn((T, V), generator=g) * sure

        def rows(y):
            wide = torch.full((T, V + pad), float("nan"), dtype=TORCH[dt] if dt != "f32" else torch.float32)
            wide[:, pad // 2:pad // 2 + V] = torch.softmax(y, -1)
            return wide.cuda()[:, pad // 2:pad // 2 + V]
        self.target = rows(x)
        self.draft = rows(x + torch.randn((T, V), generator=g) * 0.7) if drafted else None
        self.parents = [0] * before + [p for t in trees for p in t] + [0] * behind
        self.ids = torch.randint(V, (T,), generator=g)
        q = (self.draft if drafted else self.target).cpu().float()
        for s, t in zip(self.starts, trees):
            for i, p in enumerate(t):
                if 0 <= p < i:
                    self.ids[s + i] = torch.multinomial(q[s + p], 1, generator=g)[0]
        self.u, self.r = torch.rand(T, generator=g), torch.rand(len(trees), generator=g)
        self.lengths = [100 + 3 * i for i in range(len(trees))]

    def run(self, room=6, **over):
        B = len(self.r)
        path = torch.full((B, room + 3), -7, dtype=torch.int32, device="cuda")
        accepted, following, after = i32([-7] * B), i64([-7] * B), i32([-7] * B)
        a = [over.get(n, x) for n, x in (("target", self.target), ("draft", self.draft), ("ids", self.ids.cuda()), ("parents", i32(self.parents)))]
        nt.verify_tree(*a, i32(self.starts), self.u.cuda(), self.r.cuda(), path[:, 1:1 + room], accepted, following, i32(self.lengths), after)
        path = path.cpu()
        assert (path[:, 0] == -7).all() and (path[:, 1 + room:] == -7).all()
        return path[:, 1:1 + room].tolist(), accepted.tolist(), following.tolist(), after.tolist()

    def check(self, room=6):
        want = ot.verify(f64(self.target), None if self.draft is None else f64(self.draft), self.ids.tolist(), self.parents, self.starts, self.u.tolist(), self.r.tolist(), room)
        got = self.run(room)
        counts = [b - a for a, b in zip(self.starts, self.starts[1:])]
        assert got[:3] == tuple(want)
        assert got[3] == [n - c + k for n, c, k in zip(self.lengths, counts, want[1])]
        return want


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("drafted", [True, False])
@pytest.mark.parametrize("V", [1, 2, 7, 1000, 4099, 40001])
def test_verification(dt, drafted, V):
    g = np.random.default_rng(V)
    stood = 0
    for seed in range(3 if V < 40000 else 1):
        trees = [random_tree(n, g) for n in (1, 9, 0, 30, 5, 70)] + [list(range(-1, 7))]
        d = Drafts(trees, V, dt, drafted, seed, before=2, behind=1, sure=4.0 if V > 10 else 1.0, pad=seed)
        if not drafted:
            d.u *= 0.2
        stood += sum(d.check()[1]) - 6
    assert stood > 0                                                          # (some drafts, beside the six roots)
    d.check(room=1)
    d.check(room=2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("drafted", [True, False])
def test_many_children(dt, drafted):
    """Nodes with more children than are tried, over more tokens than a wavefront has lanes; the same token twice; few words so that something is left of none."""
    for V in (5, 300):
        d = Drafts([[-1] + [0] * 150, [-1, 0] + [1] * 90 + [5] * 3, [-1] + [0] * 63 + [0] * 5], V, dt, drafted, 1, sure=1.0)
        for u in (0.999, 0.5, 0.05):
            d.u.fill_(u)
            d.check()
    d = Drafts([[-1] + [0] * 70], 1000, dt, drafted, 2)                       # the 64th child stands, the 65th is not tried
    d.u.fill_(0.9999999)
    for last in (64, 65):
        d.target[0] = 0
        d.target[0, :200] = 1 / 256
        d.ids[1:] = torch.arange(300, 370)
        d.ids[last] = 3
        d.u[last] = 0.0
        want = d.check()
        assert want[1] == [2 if last == 64 else 1]


def test_borders_between_tokens():
    """Probabilities and random numbers that are short binary numbers: every comparison is exact, and ties go to the next token."""
    V = 1 << 16
    for dt in ("f32", "f16", "bf16"):
        d = Drafts([[-1]] * 64, V, dt, False)
        d.target.fill_(2.0 ** -16)
        d.r = torch.arange(64) * (1021 / 65536)
        assert d.run()[2] == [1021 * i for i in range(64)]
        d.target[:, ::2] = 0
        d.r = torch.arange(64) / 64
        assert d.run()[2] == [1024 * i + 1 for i in range(64)]
        d.target.fill_(0)
        d.target[:, 40000] = 0.5
        d.r = torch.tensor([0.0, 0.25, 0.999] + [float(np.nextafter(np.float32(1), np.float32(0)))] * 61)
        assert d.run()[2] == [40000] * 64
    # acceptance: u q m < w, not where they are equal
    d = Drafts([[-1, 0]] * 4, 4, "f32", True)
    d.ids[1::2] = 1
    d.target.copy_(torch.tensor([0.25, 0.25, 0.5, 0.0]).expand(8, 4))
    d.draft.copy_(torch.tensor([0.25, 0.5, 0.25, 0.0]).expand(8, 4))
    d.u[1::2] = torch.tensor([0.0, 0.4999, 0.5, 0.75])
    d.r.fill_(0.5)
    assert d.check()[1] == [2, 2, 1, 1]


def test_probabilities_that_are_none():
    """Rows of zeros, negative numbers, infinities and NaN count as zeros; random numbers outside [0, 1) end the row; drafts outside the vocabulary are passed over."""
    for dt in ("f32", "f16", "bf16"):
        d = Drafts([[-1, 0, 0, 1]] * 9, 3001, dt, True, 4)
        bad = torch.tensor([float("nan"), float("inf"), -1.0, -float("inf")]).to(d.target.dtype).cuda()
        for i in range(4):
            d.target[4 * i, 17] = bad[i]
            d.draft[4 * i, 18] = bad[i]
            d.target[4 * i + 1, 3000] = bad[i]
        d.target[16:20] = 0                                                   # nothing at all
        d.target[20:24] = d.draft[20:24]                                      # nothing is left where one is rejected
        d.u[20:24] = 1.5
        d.ids[24:28] = torch.tensor([5, -1, 3001, 2 ** 40])
        d.target[28:32, :3000] = 0
        want = d.check()
        assert want[2][4] == -1 and want[1][6] == 1
        d.r[:] = float("nan")
        assert all(0 <= x for x in np.array(d.run()[2])[[0, 1, 2, 3, 5, 6, 7, 8]])
        d.r[:] = 2.0
        last = d.run()
        for b in (6, 7):
            w = d.target[4 * b + last[0][b][last[1][b] - 1]].cpu()
            assert last[2][b] == int(torch.nonzero(w)[-1])


def test_verification_without_lengths_and_without_tokens():
    d = Drafts([[-1, 0], [-1]], 50)
    path, accepted, following = i32([[9] * 3] * 2), i32([9, 9]), i64([9, 9])
    nt.verify_tree(d.target, None, d.ids.cuda(), i32(d.parents), i32(d.starts), d.u.cuda(), d.r.cuda(), path, accepted, following)
    want = ot.verify(f64(d.target), None, d.ids.tolist(), d.parents, d.starts, d.u.tolist(), d.r.tolist(), 3)
    assert (path.tolist(), accepted.tolist(), following.tolist()) == tuple(want)
    e = torch.empty((0, 50), device="cuda")
    nt.verify_tree(e, None, i64([]), i32([]), i32([0, 0, 0]), e[:, 0], d.r.cuda(), path, accepted, following, i32([5, 6]), accepted)
    assert path.tolist() == [[-1] * 3] * 2 and accepted.tolist() in ([0, 0], [5, 6]) and following.tolist() == [-1, -1]
    nt.verify_tree(d.target[:, :0], None, d.ids.cuda(), i32(d.parents), i32(d.starts), d.u.cuda(), d.r.cuda(), path, accepted, following)
    assert accepted.tolist() == [1, 1] and following.tolist() == [-1, -1]


# ------------------------------------------------------------------------------------------------------------ moving what stands
@pytest.mark.parametrize("kind", ["f16", "bf16", "e4m3", "i8"])
@pytest.mark.parametrize("heads,size,page,layout,layers", [(2, 64, 16, "dense", 1), (3, 128, 7, "heads first", 3), (1, 8, 1, "dense", 2), (5, 80, 24, "padded", 2), (2, 256, 16, "dense", 40)])
def test_what_stands_is_moved(kind, heads, size, page, layout, layers):
    g = np.random.default_rng(size)
    past, new = [0, 5, 33, 100, 7, 20], [9, 64, 12, 1, 30, 0]
    paths = [[0, 1, 2, 5, 8], sorted(g.choice(64, 30, replace=False)), [0, 2, 3, 4, 5, 6, 11], [0], [0, 29], []]
    room = max(map(len, paths)) + 1
    path = np.array([[*p] + [-1] * (room - len(p)) for p in paths])
    need = [-(-(a + b) // page) for a, b in zip(past, new)]
    table = np.full((6, max(need) + 1), -1, np.int64)
    order, at = g.permutation(sum(need) + 2), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    caches, want = [], []
    for layer in range(layers):
        c = empty_cache(sum(need) + 2, page, heads, size, kind, layout)
        for t in c:
            if t is not None:
                shape = t.shape
                t.view(torch.uint8 if t.element_size() == 1 else t.dtype).copy_((torch.randn(shape) * 50).to(torch.uint8 if t.element_size() == 1 else t.dtype))
        caches.append(c if c[2] is not None else c[:2])
        want.append([raw(t).numpy().copy() for t in caches[-1]])
    lengths, accepted = [a + len(p) for a, p in zip(past, paths)], [len(p) for p in paths]
    wide = i32(np.full((6, room + 2), 3))
    wide[:, 1:1 + room] = i32(path)
    nt.cache_compact(caches, i32(table), i32(lengths), wide[:, 1:1 + room], i32(accepted))
    torch.cuda.synchronize()
    for c, w in zip(caches, want):
        for t, x in zip(c, w):
            ot.compact(x, table, np.array(lengths), path, np.array(accepted))
            assert np.array_equal(raw(t).numpy(), x)


def test_moves_that_are_none():
    """Paths that do not ascend move within bounds; entries at or below their place, positions before 0, pages that are missing, counts beyond the path's room."""
    c = [empty_cache(6, 4, 2, 64, "f16") for _ in range(2)]
    for k, v, *_ in c:
        k.copy_(torch.randn(k.shape))
        v.copy_(torch.randn(v.shape))
    table = np.array([[0, 1, -1], [2, 1 << 30, 3], [4, 5, -2 ** 31]])
    for lengths, path, accepted in (([6, 6, 6], [[0, -5, 1], [0, 1, 2], [-1, -1, -1]], [3, 3, 3]),                     # nothing moves
                                    ([2, 2, 2], [[4, 5, 6]] * 3, [9, 9, 9]), ([5, 2 ** 31 - 1, -2 ** 31], [[0, 2 ** 31 - 1, -2 ** 31]] * 3, [3, 2, 1]),
                                    ([7, 6, 6], [[0, 7, 100], [0, 2, 5], [0, 100, 2 ** 30]], [2, 3, 3]), ([0, 0, 0], [[1, 2, 3]] * 3, [0, -1, -2 ** 31])):
        want = [[raw(t).numpy().copy() for t in x[:2]] for x in c]
        nt.cache_compact([x[:2] for x in c], i32(table), i32(lengths), i32(path), i32(accepted))
        for x, w in zip(c, want):
            for t, y in zip(x[:2], w):
                ot.compact(y, table, np.array(lengths), np.array(path), np.maximum(np.array(accepted), -2 ** 31))
                assert np.array_equal(raw(t).numpy(), y)


# ------------------------------------------------------------------------------------------------------------ every way, graphs, streams
def calls(seed=0, cls=None, stream=None, **k):
    """One call of each operator; returns what they gave."""
    f = (lambda t: t.as_subclass(cls)) if cls else (lambda t: t)
    b = Trees([(9, 3000), (20, 40)], 4, 2, 64, 16, "f16", "i8", seed=seed)
    out = [f(b.q) if cls else b.q]
    got = [b.run(q=out[0], max_queries=20, stream=stream)]
    p = [i32([40, 3]), i32([5, 17]), 16, i32(np.full((2, 9), -1)), i32([0, 0]), i32(np.arange(30)), i32([30]), i32([0] * 3), i32([0] * 2), i64([0] * 30), i32([0] * 30)]
    nt.cache_fit(f(p[0]), *p[1:], stream=stream)
    m, d = torch.zeros((9, 2), dtype=torch.int64, device="cuda"), i32([0] * 9)
    at = i32([0] * 9)
    nt.tree_masks(f(i32([-1, 0, 0, 1, 2, 2, -1, 0, 1])), i32([0, 6, 9]), m, d, i32([20, 30]), at, window=2, stream=stream)
    v = Drafts([random_tree(12, np.random.default_rng(seed)), [-1, 0, 1]], 5000, seed=seed)
    path, accepted, following, after = i32([[0] * 5] * 2), i32([0, 0]), i64([0, 0]), i32([0, 0])
    nt.verify_tree(f(v.target), v.draft, v.ids.cuda(), i32(v.parents), i32(v.starts), v.u.cuda(), v.r.cuda(), path, accepted, following, i32([50, 60]), after, stream=stream)
    nt.cache_compact([(f(b.c[0]), *b.c[1:])], i32(b.table), i32([2994, 22]), i32([[0, 2, 8], [0, 19, 0]]), i32([3, 2]), stream=stream)
    return [every_byte(t) for t in (*got, *p[3:], m, d, at, path, accepted, following, after, *b.c)]


def test_every_way_gives_the_same_bits():
    want = calls()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    others = [calls(cls=Tagged), calls(stream=torch.cuda.current_stream())]
    with torch.cuda.stream(side):
        others.append(calls())
    torch.cuda.synchronize()
    for o in others:
        assert all(torch.equal(x, y) for x, y in zip(o, want))


def test_errors_of_arguments():
    b = Trees([(3, 30)], 4, 2, 64, 16, "f16", "e4m3")
    a = list(b.args())
    for i, wrong in ((3, a[3].long()), (4, a[4].long()), (4, a[4][:1]), (5, i32([1, 2])), (6, a[6].int()), (6, a[6][:, 0]), (7, a[7].float()), (8, None)):
        with pytest.raises(ValueError):
            nt.sdpa_paged_tree(*a[:i], wrong, *a[i + 1:])
    with pytest.raises(ValueError):
        nt.sdpa_paged_tree(*a, depths=i32([1]), window=3)
    with pytest.raises(nt.NtError):
        nt.sdpa_paged_tree(*a, window=3)
    with pytest.raises(nt.NtError):
        nt.sdpa_paged_tree(*a[:6], a[6][:2], *a[7:])
    nt.sdpa_paged_tree(*a)
    p = [i32([4]), i32([5]), 16, i32([[-1, -1]]), i32([0]), i32([0, 1]), i32([2]), i32([0, 0]), i32([0]), i64([0] * 5), i32([0] * 5)]
    for i, wrong in ((0, i32([4, 4])), (1, i64([5])), (3, i32([1, 2])), (4, i32([0, 0])), (5, i64([0, 1])), (6, i32([1, 2])), (7, i32([0])), (8, i64([0])), (9, i32([0] * 5)), (10, i32([0] * 4))):
        with pytest.raises(ValueError):
            nt.cache_fit(*p[:i], wrong, *p[i + 1:])
    with pytest.raises(nt.NtError):
        nt.cache_fit(*p[:2], 0, *p[3:])
    nt.cache_fit(*p)
    m = torch.zeros((3, 1), dtype=torch.int64, device="cuda")
    t = [i32([-1, 0, 0]), i32([0, 3]), m, i32([0] * 3)]
    for i, wrong in ((0, i32([0, 0])), (1, i64([0, 3])), (1, i32([])), (2, m.int()), (2, m[:, 0]), (3, i32([0]))):
        with pytest.raises(ValueError):
            nt.tree_masks(*t[:i], wrong, *t[i + 1:])
    with pytest.raises(ValueError):
        nt.tree_masks(*t, lengths=i32([3]))
    with pytest.raises(nt.NtError):
        nt.tree_masks(*t, window=-1)
    d = Drafts([[-1, 0]], 50)
    v = [d.target, d.draft, d.ids.cuda(), i32(d.parents), i32(d.starts), d.u.cuda(), d.r.cuda(), i32([[0, 0]]), i32([0]), i64([0])]
    for i, wrong in ((0, d.target[0]), (1, d.draft.half()), (2, v[2].int()), (3, i64([0, 0])), (4, i32([0])), (5, v[5].double()), (6, v[6][:0]), (7, i32([0])), (8, i64([0])), (9, i32([0]))):
        with pytest.raises(ValueError):
            nt.verify_tree(*v[:i], wrong, *v[i + 1:])
    with pytest.raises(ValueError):
        nt.verify_tree(*v, i32([5]))
    with pytest.raises(nt.NtError):
        nt.verify_tree(d.target, d.draft[:, :49], *v[2:])
    nt.verify_tree(*v)
    c = [(b.c[0], b.c[1], b.c[2], b.c[3]), i32(b.table), i32([30]), i32([[0, 2]]), i32([2])]
    for i, wrong in ((1, i64(b.table)), (2, i32([1, 2])), (3, i32([0, 2])), (4, i64([2]))):
        with pytest.raises(ValueError):
            nt.cache_compact([c[0]], *[wrong if j == i else x for j, x in enumerate(c) if j])
    with pytest.raises(nt.NtError):
        nt.cache_compact([c[0], c[0][:2]], *c[1:])
    with pytest.raises(ValueError):
        nt.cache_compact([(c[0][0], c[0][1], c[0][2], None)], *c[1:])
    nt.cache_compact([c[0]], *c[1:])


def test_captured_into_a_graph():
    """A step of all five, replayed on changing inputs with eager calls of the same kind between."""
    b = Trees([(9, 2000), (9, 60)], 4, 2, 64, 16, "f16", "e4m3")
    table, starts, lengths, out = i32(b.table), i32(b.starts), i32(b.lengths), torch.empty_like(b.q)
    parents, masks, depths, positions = i32([-1, 0, 0, 1, 1, 2, 4, 4, 7] * 2), torch.zeros((18, 1), dtype=torch.int64, device="cuda"), i32([0] * 18), i32([0] * 18)
    v = Drafts([[-1, 0, 0, 1, 1, 2, 4, 4, 7]] * 2, 40000, seed=3)
    ids, u, r = v.ids.cuda(), v.u.cuda(), v.r.cuda()
    zero, pages = i32([0, 0]), b.c[0].shape[0]

    def step(o):
        # (a pool of its own, so that every replay begins with the same)
        pool = [torch.full((2, 200), -1, dtype=torch.int32, device="cuda"), torch.zeros_like(zero), torch.arange(pages, dtype=torch.int32, device="cuda"), torch.full_like(zero[:1], pages)]
        got = [torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros_like(zero), torch.zeros(4500, dtype=torch.int64, device="cuda"), torch.zeros(4500, dtype=torch.int32, device="cuda")]
        nt.cache_fit(zero, lengths, 16, *pool, *got)
        nt.tree_masks(parents, starts, masks, depths, lengths, positions)
        nt.sdpa_paged_tree(b.q, b.c[0], b.c[1], table, starts, lengths, masks, o, b.c[2], b.c[3], max_queries=9)
        path, accepted, following, after = (torch.zeros(s, dtype=t, device="cuda") for s, t in (((2, 5), torch.int32), ((2,), torch.int32), ((2,), torch.int64), ((2,), torch.int32)))
        nt.verify_tree(v.target, v.draft, ids, parents, starts, u, r, path, accepted, following, lengths, after)
        cache = [t.clone() for t in b.c]
        nt.cache_compact([tuple(cache)], table, after, path, accepted)
        return [o, *pool, *got, masks, positions, path, accepted, following, after, *cache]
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = step(out)
    for i in range(4):
        b.q.copy_(normal(b.q.shape, "f16", 30 + i))
        u.copy_(torch.rand(18, generator=torch.Generator().manual_seed(i)))
        r.copy_(torch.rand(2, generator=torch.Generator().manual_seed(i + 9)))
        lengths.copy_(i32([2000 - 100 * i, 60 - i]))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [every_byte(t) for t in made]
        want = [every_byte(t) for t in step(torch.empty_like(out))]
        assert all(torch.equal(x, y) for x, y in zip(got, want))
        step(torch.empty_like(out))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(every_byte(x), y) for x, y in zip(made, want))


def test_two_streams():
    """Shares of calls on two streams meet in the workspace."""
    bs = [Trees([(9, 3500), (3, 2000)], 4, 2, 64, 16, "f16", seed=s) for s in (1, 2)]
    ds = [Drafts([random_tree(9, np.random.default_rng(s))] * 3, 50000, seed=s) for s in (1, 2)]
    want = [b.run(max_queries=9).clone() for b in bs]
    want_v = [d.run() for d in ds]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    got, got_v = [[], []], [[], []]
    for _ in range(10):
        for i, (b, d, s) in enumerate(zip(bs, ds, streams)):
            with torch.cuda.stream(s):
                got[i].append(b.run(max_queries=9))
                got_v[i].append(d.run())
    torch.cuda.synchronize()
    assert all(torch.equal(x, w) for g, w in zip(got, want) for x in g)
    assert all(x == w for g, w in zip(got_v, want_v) for x in g)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_small_weights_are_not_off_to_one_side(dt):
    """One key with 70 % of a row, 131072 others of some 2^-18 each, all of one program (more sequences than are dealt out): a weight's error has no side that adds up over the keys.

    V is 1, so that what the scores are off by cancels.  A weight multiplies V as two numbers, rounded to nearest or raised by 2^-32 of the largest (2^-16 of itself in bf16): n 2^-32, or 2^-17
    on its side.  fp32 sums of n numbers, their roundings of either sign: 6 sqrt(n) 2^-24 for six times their spread.  The result's rounding: half a step."""
    n, size = 131072, 64
    b = Trees([(1, n)] + [(0, 0)] * 1024, 1, 1, size, 1024, dt, seed=7)
    q, first = b.q[0, 0].double(), int(b.table[0, 0])
    k = b.c[0][torch.tensor(b.table[0, :n // 1024], device="cuda")].double().view(n, size)
    rest = torch.exp((k[1:] @ q) / 8).sum().item()
    b.c[0][first, 0, 0] = (q * (np.log(rest * 0.7 / 0.3) * 8 / (q @ q).item())).to(TORCH[dt])
    b.c[1].fill_(1.0)
    got = f64(b.run(max_queries=1))
    h = torch.finfo(TORCH[dt]).eps / 2
    assert np.abs(got - 1).max() <= h + 6 * n ** 0.5 * 2.0 ** -24 + (n * 2.0 ** -32 if dt == "f16" else 2.0 ** -17)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("size", [64, 128, 256])
def test_infinities_with_small_weights(dt, size):
    """An infinity that every row sees at a weight of e^-20 of the largest, in the same block, stays one."""
    for bad in (float("inf"), -float("inf")):
        b = Trees([(5, 400), (3, 90)], 2, 1, size, 16, dt, seed=2)
        b.q.fill_(1.0)
        b.c[0][int(b.table[0, 0]), 3] = 20 * size ** -0.5
        want = b.run().clone()
        b.check(want)
        b.c[1][int(b.table[0, 1]), 4, 0, 7] = bad
        got = b.run()
        hit = torch.zeros_like(got, dtype=torch.bool)
        hit[:5, :, 7] = True
        assert torch.equal(got[~hit], want[~hit]) and (got[hit] == bad).all()


def sums_at_a_border(g, tiny):
    """256 sums of chunks, four to a lane: added lane by lane and then by a scan, what is ahead of some lane comes out above the run to the end of the lane before it, and half of all lies between.
    `tiny`: of that lane's first chunk."""
    def scanned(v):
        mine = ((v[:, 0] + v[:, 1]) + v[:, 2]) + v[:, 3]
        upto, d = mine.copy(), 1
        while d < 64:
            upto[d:] = upto[d:] + upto[:-d]
            d *= 2
        return mine, upto
    while True:
        v = np.zeros((64, 4))
        lane = int(g.integers(3, 50))
        v[:lane] = np.exp2(g.uniform(-40, 0, (lane, 4))).astype(np.float32)
        v[lane, 0] = tiny
        mine, upto = scanned(v)
        run = upto[lane - 1] - mine[lane - 1]
        for x in v[lane - 1]:
            run = run + x
        left = run
        for i in range(3):                                                    # as much again, in three numbers of 32 bits
            v[60, i] = np.float32(left) if np.float32(left) <= left else np.nextafter(np.float32(left), np.float32(0))
            left -= v[60, i]
        if run <= 0.5 * scanned(v)[1][63] < upto[lane] - mine[lane]:
            return v.reshape(-1)


@pytest.mark.parametrize("V,tiny", [(256 * 1024, 0.0), (256 * 8192, 2.0 ** -90)])
def test_goals_between_two_sums(V, tiny):
    """The next token has a weight also where the random number falls between two sums of the same numbers, added in another order."""
    g, V = np.random.default_rng(3), V
    d = Drafts([[-1]], V, "f32", False)
    d.r.fill_(0.5)
    for _ in range(20):
        w = np.zeros((256, V // 256))
        w[:, -1] = sums_at_a_border(g, tiny)
        w = w.reshape(-1)
        d.target.copy_(torch.from_numpy(w)[None])
        token = d.run()[2][0]
        upto = np.cumsum(w)
        assert w[token] > 0 and upto[token] - w[token] <= upto[-1] * (0.5 + 1e-12) and upto[token] >= upto[-1] * (0.5 - 1e-12)


@pytest.mark.parametrize("V", [4, 20001, 200003])
def test_what_is_left_is_a_quotient(V):
    """w / m - q where w / m is exactly q: nothing is left, and the next token is the target's.  (1 / m, rounded, is above it: with the product something would be left.)"""
    d = Drafts([[-1, 0, 0] + [1] * 7] * 2, V, "f32", True)
    d.target.fill_(0)
    d.draft.fill_(0)
    q, m = 3 / 32, 91 / 2 ** 14
    assert q * m * (1 / m) > q
    d.draft[:, 0], d.draft[:, 1], d.draft[:, 2], d.draft[:, 3] = q, 1 - q, 0.5, 0.75
    d.target[:, 0], d.target[:, 1], d.target[:, 3] = q + q * m, (1 - q) + (1 - q) * m, 0.5
    d.ids.fill_(2)
    d.r[:] = torch.tensor([0.99, 0.1])
    want = d.check()
    assert want[1:] == ([1, 1], [3, 1])


def test_more_streams_than_workspaces():
    """Calls of five streams, none waited for by the host: the attention's shares (34 MB) meet in the one large piece of the workspace, the verification's states and sums in three small ones."""
    bs = [Trees([(9, 3500), (3, 2000 + 100 * s)], 4, 1, 128, 16, "f16", seed=s) for s in range(5)]
    ds = [Drafts([random_tree(9, np.random.default_rng(s))] * 3, 50000, seed=s) for s in range(5)]
    calls = []
    for b, d in zip(bs, ds):
        a, ids, parents, starts, u, r, lengths = b.args(), d.ids.cuda(), i32(d.parents), i32(d.starts), d.u.cuda(), d.r.cuda(), i32(d.lengths)

        def call(out, path, accepted, following, after, a=a, d=d, v=(ids, parents, starts, u, r), lengths=lengths):
            nt.sdpa_paged_tree(*a[:7], out, *a[8:], max_queries=9)
            nt.verify_tree(d.target, d.draft, *v, path, accepted, following, lengths, after)
        calls.append(call)

    def outputs(b):
        return torch.full_like(b.q, -5.0), i32([[-7] * 6] * 3), i32([-7] * 3), i64([-7] * 3), i32([-7] * 3)
    want, got = [outputs(b) for b in bs], [[outputs(b) for _ in range(20)] for b in bs]
    for call, o in zip(calls, want):
        call(*o)
        torch.cuda.synchronize()
    for b, d, o in zip(bs, ds, want):
        b.check(o[0])
        assert (o[1].tolist(), o[2].tolist(), o[3].tolist(), o[4].tolist()) == d.run()
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    for i in range(20):
        for call, o, s in zip(calls, got, streams):
            with torch.cuda.stream(s):
                call(*o[i])
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        assert all(torch.equal(x, y) for o in runs for x, y in zip(o, w))
