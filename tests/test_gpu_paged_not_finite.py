"""Attention over an 8-bit paged cache: a value that is not a number, at a key whose weight is nothing in 32 bits.

Such a value lies in its scale alone (its codes are 0).  A row that sees the key shows it however small the weight is, and wherever the row's blocks of keys
begin; one that does not see it has no part of it."""
import pytest
import torch

import paper_2507_11978_amd as nt
from test_gpu_paged import Batch, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["e4m3", "i8"])
@pytest.mark.parametrize("size", [64, 128, 256])
@pytest.mark.parametrize("infinitely", [False, True])
def test_a_weight_of_nothing_does_not_hide_nan(dt, kind, size, infinitely):
    for seqs, hints, at in (([(100, 130)], 0, 20), ([(100, 130)], 0, 70), ([(1, 40), (90, 2000)], 0, 1950), ([(4, 40)], 4, 20), ([(4, 40)], 4, 38), ([(2, 3000)], 2, 2998)):
        b = Batch(seqs, 1, 1, size, 16, dt, kind, seed=3)
        last = len(seqs) - 1
        b.q[..., 0] = 8.0
        k, v = torch.zeros(1, 1, size, dtype=b.q.dtype), normal((1, 1, size), dt, 5)
        k[..., 0] = -1.0 if infinitely else -15.0 * size ** 0.5              # (a score of -120)
        v[..., 7] = float("nan")
        page, place = int(b.table[last, at // 16]), at % 16
        nt.cache_write(k.cuda(), v.cuda(), torch.tensor([page * 16 + place]).cuda(), *b.c)
        if infinitely:
            b.c[2][page, place] = 3e38                                      # (beyond 32 bits)
        got = b.run(max_queries=hints)
        b.check(got, f"{seqs} {at}")
        first = b.starts[last] + max(0, at - (seqs[last][1] - seqs[last][0]))
        assert torch.isnan(got[first:]).all() and torch.isfinite(got[:first]).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("size", [64, 80, 128, 256])
@pytest.mark.parametrize("q_heads,new", [(1, 1), (4, 1), (6, 3), (16, 2)])
def test_infinite_values_that_every_row_sees(dt, size, q_heads, new):
    """A 16-bit cache: a seen infinity makes the element it lies in infinite, two of opposite sign or NaN make it NaN, and the others are what they are."""
    inf = float("inf")
    for seqs, hints in (([(new, 300), (new, 200)], (new, 300)), ([(new, 6000)], (new, 6000))):
        b = Batch(seqs, q_heads, 1, size, 16, dt, seed=6)
        want = b.run(max_queries=hints[0], max_length=hints[1]).clone()
        for places in (((20, 3, inf),), ((20, 3, -inf), (21, 5, inf)), ((20, 3, inf), (150, 3, -inf)), ((20, 3, float("nan")), (40, 5, inf), (130, 5, inf))):
            was = [b.c[1][int(b.table[0, at // 16]), at % 16, 0, d].clone() for at, d, _ in places]
            for at, d, x in places:
                b.c[1][int(b.table[0, at // 16]), at % 16, 0, d] = x
            got = b.run(max_queries=hints[0], max_length=hints[1])
            torch.cuda.synchronize()
            assert nt.last_paged_plan().rows == (16 if q_heads * new <= 16 else 32 if size <= 128 else 128)
            expected = want.clone()
            expected[:b.starts[1], :, [d for _, d, _ in places]] = 0
            for at, d, x in places:
                expected[:b.starts[1], :, d] += x
            assert torch.equal(torch.nan_to_num(got, 7.0, 8.0, 9.0), torch.nan_to_num(expected, 7.0, 8.0, 9.0))
            for (at, d, _), x in zip(places, was):
                b.c[1][int(b.table[0, at // 16]), at % 16, 0, d] = x
