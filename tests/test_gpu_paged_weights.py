"""How exactly the paged attention's weights count, against the fp64 oracle.

Bounds.  The result's rounding: h |O| with h = eps / 2 of its type (fp16: 2^-25 at least).  A score is an fp32 sum of `size` products, some eight more roundings
follow until its exponential: off by 2^-24 (size + 8) S at most, with S the largest of scale * sum |q| |k| over the row's keys; that is the relative
error of a weight, and twice that of the quotient.  Sums over n keys in fp32: 2^-24 (n + 16).  What the weights are rounded to before they multiply V: in two
parts of bf16 2^-17 (the rest's rounding; in the mean over a row's keys half of it at most, 2^-18), in two of fp16 2^-23 and the spacing of its smallest numbers, 2^-25 of a weight of 1 for each key.
All of these but the first are relative to A = sum_j p_j |V_j|, the last to the largest |V|."""
import numpy as np
import pytest
import torch

import paper_2507_11978_amd as nt
from oracle import paged as op
from test_gpu_paged import KINDS, TORCH, Batch, f64, normal

pytestmark = pytest.mark.gpu


def check(b, got, what):
    k, v = b.values()
    q, got = f64(b.q), f64(got)
    ref, A, _ = op.attend(q, k, v, b.table, b.starts, b.lengths)
    S = np.zeros(A.shape[:2] + (1,))
    for s, n in enumerate(b.lengths):
        at = np.arange(n)
        rows = np.abs(k[b.table[s, at // b.page], at % b.page])               # [keys, heads, size]
        mine = slice(b.starts[s], b.starts[s + 1])
        group = q.shape[1] // rows.shape[1]
        for h in range(q.shape[1]):
            S[mine, h, 0] = (np.abs(q[mine, h]) @ rows[:, h // group].T).max(1) / np.sqrt(q.shape[2])
    n, h = max(b.lengths), torch.finfo(TORCH[b.dt]).eps / 2
    tol = 1.01 * h * np.abs(ref) + A * (2.0 ** -24 * (2 * (q.shape[2] + 8) * S + n + 16) + 1.01 * 2.0 ** -18)
    if b.dt == "f16":
        tol += 2.0 ** -25
    if b.kind == "f16":
        tol += 2.0 ** -25 * n * np.abs(v[np.isfinite(v)]).max()
    worst = (np.abs(got - ref) - tol).max()
    assert worst <= 0, f"{what}: {worst:.3g} over the bound, {(np.abs(got - ref) / tol).max():.3g} times"


@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("size", [64, 128, 256])
@pytest.mark.parametrize("value", [2.0 ** -4, 2.0 ** -10])
@pytest.mark.parametrize("raised", [False, True])
def test_a_large_value_that_weighs_nothing(kind, size, value, raised):
    """fp16 queries over codes: a key with values near the type's largest and a weight of e^-25.6 beside the others', which have ordinary ones.  `raised`: it
    weighs more than the keys before it, until others follow."""
    for seqs, hints, at in (([(40, 300)], 0, 3), ([(40, 300)], 0, 200), ([(40, 300)], 0, 280), ([(64, 2000)], 0, 1000), ([(4, 200)], 4, 3), ([(4, 200)], 4, 150), ([(2, 3000)], 2, 1500)):
        b = Batch(seqs, 2, 1, size, 16, "f16", kind, seed=4, poison=False)
        n = seqs[0][1]
        slots = torch.tensor([int(b.table[0, j // 16]) * 16 + j % 16 for j in range(n)])
        k, v = normal((n, 1, size), "f16", 6), normal((n, 1, size), "f16", 7, value)
        b.q[..., 0] = 8.0
        k[:, :, 0] = 3.2 * size ** 0.5 if raised else 0.0
        k[at, :, 0] -= 3.2 * size ** 0.5
        if raised:
            k[:at, :, 0] = -3.2 * size ** 0.5
        v[at] = torch.where(v[at] < 0, -6e4, 6e4)
        nt.cache_write(k.cuda(), v.cuda(), slots.cuda(), *b.c)
        got = b.run(max_queries=hints, max_length=hints and n)
        torch.cuda.synchronize()
        assert nt.last_paged_plan().rows == (16 if hints else 128)
        check(b, got, f"{seqs} {at}")


@pytest.mark.parametrize("dt,kind", KINDS)
@pytest.mark.parametrize("q_heads,heads,size,page", [(1, 1, 64, 16), (8, 2, 128, 16), (6, 6, 80, 24), (4, 2, 256, 16), (20, 1, 120, 16)])
def test_few_rows_round_the_result_only(dt, kind, q_heads, heads, size, page):
    """One token of each sequence, or a few: reading K and V takes the time, the weights keep their bits."""
    for seqs, length, shared in (([(1, 1), (1, 17), (1, 64), (1, 300)], 0, False), ([(1, 3000), (1, 40)], 3000, True)):
        b = Batch(seqs, q_heads, heads, size, page, dt, kind, seed=2)
        got = b.run(max_queries=1, max_length=length)
        torch.cuda.synchronize()
        p = nt.last_paged_plan()
        held = length * size * 2 * (1 if kind in ("e4m3", "i8") else 2)       # of K and V to a head (shared from 384 KB on)
        assert p.rows < 128 and (p.shares > 1) >= (shared and held >= 384 << 10)
        check(b, got, f"{seqs}")
