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
